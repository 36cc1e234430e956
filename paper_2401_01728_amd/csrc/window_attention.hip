// Causal attention over a sliding window and a few first keys, forward and backward: bf16 operands, fp32 scores, softmax statistics and sums.
//
//   token t of a sequence is at position p = start + t and sees key j where  j <= p  and  (j > p - window  or  j < sinks)
//   s = q k^T / sqrt(dh),  P = softmax over the keys that a token sees,  o = P v
//   dv = P^T do,  ds = P (do v^T - rowsum(do o)),  dq = ds k / sqrt(dh),  dk = ds^T q / sqrt(dh)
//
// Keys may lie in a cache of Sk rows that is a ring behind its sinks: key j in row j below Sk, further ones in sinks + (j - sinks) % (Sk - sinks).
// A key whose row a later one has taken is seen by nobody.
//
// The `share` query heads of a key/value head are taken as ONE list of rows, row r being head r % share of token r / share: the rows of a workgroup
// are then few tokens, whose windows nearly coincide, and a key/value head is read once for all heads that share it.
// As in cross_attention.hip a wave owns 32 rows (or keys), which are the lanes, and the other side streams through LDS in tiles of 64.  The keys of
// a workgroup's rows are the sinks and ONE range that begins at the oldest key of its first token: tiles begin there, so that a range of w keys and
// the few tokens' own is cut into as few tiles as there can be, and a tile never holds a key that nobody sees.  Only tiles that hold a row's
// border are masked, by selects behind a branch.
#include <math.h>
#include "../../include/rv_kernels.h"
#include "attention_core.h"

namespace {

struct WinArgs {
  const uint16_t* q; const uint16_t* k; const uint16_t* v;
  int64_t ldq, ldk, ldv;
  const int* start; const int* length;   // device [B] or null
  uint16_t* out; int64_t ldo;
  float* lse2;                           // [B][H][Sq]
  // backward
  const uint16_t* o; const uint16_t* dout; int64_t lddo;
  uint16_t* dq; uint16_t* dk; uint16_t* dv;
  int64_t lddq, lddk, lddv;
  float* stat_lse; float* stat_d;        // [B][Hkv][Rp], in the order of the list
  float* part; float2* part_ml;          // forward: sums of the parts
  float* q_part; float* kv_part; float* sink_part;   // backward
  int B, Sq, Sk, share, Hkv, R, Rp, kv_grid, sink_grid;
  int sink_blocks, sink_parts;           // workgroups of the sinks, or 0: where no window leaves them they are keys like others
  int window, sinks, ring;               // sinks < Sk, ring = Sk - sinks
  Grid fwd, bq, bkv;
  float c2, scale;                       // log2(e) / sqrt(dh), 1 / sqrt(dh)
};

__device__ __forceinline__ int live_at(const WinArgs& a, int b) {
  if (!a.length) return a.Sq;
  const int n = a.length[b];
  return n < 0 ? 0 : n < a.Sq ? n : a.Sq;
}
__device__ __forceinline__ int live_of(const WinArgs& a, int b) { return __builtin_amdgcn_readfirstlane(live_at(a, b)); }   // (b: wave-uniform)
__device__ __forceinline__ int start_of(const WinArgs& a, int b) {
  if (!a.start) return 0;
  const int s = __builtin_amdgcn_readfirstlane(a.start[b]);
  return s < 0 ? 0 : s;
}
// row r of the list of (b, h) in a matrix of tokens whose rows are ld apart
template <int DH>
__device__ __forceinline__ int64_t row_at(const WinArgs& a, int b, int h, int r, int64_t ld) {
  const int t = r / a.share, g = r - t * a.share;
  return ((int64_t)b * a.Sq + t) * ld + (h * a.share + g) * DH;
}
__device__ __forceinline__ int64_t lse_at(const WinArgs& a, int b, int h, int r) {
  const int t = r / a.share, g = r - t * a.share;
  return ((int64_t)b * a.Hkv * a.share + h * a.share + g) * a.Sq + t;
}

// The keys that tokens ta .. tb of a sequence see, as tiles of T: first the sinks, where the window has left them, then the range from its first key
// on, from which positions are counted here.
struct Walk {
  int sink_tiles, tiles;
  int row0, span;                        // row of the range's first key; its keys
  int shift, first;                      // position of token 0; keys of the range that are sinks
  int start;                             // position of token 0 from key 0 on, no more than the sinks
};
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <int T>
__device__ __forceinline__ Walk walk_of(const WinArgs& a, int start, int n, int ta, int tb) {
  // counted from position start: the oldest key of token ta, of those whose rows have not been taken
  const int reach = ta - a.window + 1, held = n - a.ring, low = reach < held ? held : reach;
  const bool apart = start > a.sinks - low;                       // (start + low > sinks, without overflow)
  Walk w;
  w.shift = uniform(apart ? -low : start);
  w.first = apart ? 0 : a.sinks;
  w.start = start < a.sinks ? start : a.sinks;
  w.sink_tiles = apart ? (a.sinks + T - 1) / T : 0;
  w.span = uniform(tb + 1 + w.shift > 0 ? tb + 1 + w.shift : 0);
  w.tiles = uniform(w.sink_tiles + (w.span + T - 1) / T);
  const unsigned key = apart ? (unsigned)start + (unsigned)low : 0u;      // below 2^32
  w.row0 = uniform((int)(key < (unsigned)a.Sk ? key : a.sinks + (key - a.sinks) % (unsigned)a.ring));
  return w;
}
struct Tile { int row, keys; };                                   // its first key's row, and how many there are
template <int T>
__device__ __forceinline__ Tile tile_of(const WinArgs& a, const Walk& w, int i) {
  Tile t;
  const bool sink = i < w.sink_tiles;
  const int off = (sink ? i : i - w.sink_tiles) * T, left = (sink ? a.sinks : w.span) - off;
  t.row = (sink ? 0 : w.row0) + off;
  if (!sink && t.row >= a.Sk) t.row -= a.ring;
  t.keys = left < T ? left : T;
  return t;
}
// What a wave sees of the tile's keys from one on: numbers that are the wave's, so that a tile of which all of it sees all costs comparisons alone.
struct Edge {
  int at;                                // that key, counted as the others are: in the range (or among the sinks)
  int up_first, up_last;                 // the last key that the wave's first token sees, and its last one
  int reach;                             // keys that a token sees up to its last one
  int sinks;                             // keys in front of this one are seen from everywhere
  bool sink;
};
template <int T>
__device__ __forceinline__ Edge edge_of(const WinArgs& a, const Walk& w, int i, int at, int first, int last) {
  Edge e;
  e.sink = i < w.sink_tiles;
  e.at = (e.sink ? i : i - w.sink_tiles) * T + at;
  // (a token in front of the last sink has the range apart where its own row has been taken)
  const int top = a.sinks - 1;
  e.up_first = e.sink ? (w.start + first < top ? w.start + first : top) : first + w.shift;
  e.up_last = e.sink ? (w.start + last < top ? w.start + last : top) : last + w.shift;
  e.reach = e.sink ? a.sinks : a.window;
  e.sinks = e.sink ? 0 : w.first;
  return e;
}
// of the 32 keys from AT on: nobody sees any; some are ahead of a token; some are behind one
template <int AT>
__device__ __forceinline__ bool none(const Edge& e) {
  return e.at + AT > e.up_last || (e.at + AT + 31 <= e.up_first - e.reach && e.at + AT >= e.sinks);
}
template <int AT>
__device__ __forceinline__ bool ahead(const Edge& e) { return e.at + AT + 31 > e.up_first; }
template <int AT>
__device__ __forceinline__ bool behind(const Edge& e) { return e.at + AT <= e.up_last - e.reach && e.at + AT + 32 > e.sinks; }
// Which rows, counted from a tile's first, a lane sees: x <= up and (x > low or x < first).  The three are less 4 (lane / 32), so that the rows of a lane's
// registers (acc_row) are compared as constants: kept, they would be 16 registers or 32.
struct Limits { int up, low, first; };
__device__ __forceinline__ Limits limits(const WinArgs& a, const Walk& w, const Edge& e, int t) {
  const int from = e.at + ((threadIdx.x & 32) >> 3), top = a.sinks - 1;
  const int up = (e.sink ? (w.start + t < top ? w.start + t : top) : t + w.shift) - from;
  return {up, up - e.reach, e.sinks - from};
}
__device__ __forceinline__ bool sees(const Limits& s, int x) { return x <= s.up && (x > s.low || x < s.first); }
// hide(register) for what a lane does not see of 32 rows: what is ahead of it, what is behind, both where sinks are among them.
// (All comparisons first would take the scalar registers that the walk is kept in.)
template <int AT, typename Hide>
__device__ __forceinline__ void mask_ahead(int up, Hide hide) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (AT + acc_row(r, 0) > up) hide(r);
    if (r % 2) __builtin_amdgcn_sched_barrier(0);
  }
}
template <int AT, typename Hide>
__device__ __forceinline__ void mask_behind(int low, Hide hide) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (AT + acc_row(r, 0) <= low) hide(r);
    if (r % 2) __builtin_amdgcn_sched_barrier(0);
  }
}
template <int AT, typename Hide>
__device__ __forceinline__ void mask_all(const Limits& s, Hide hide) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (!sees(s, AT + acc_row(r, 0))) hide(r);
    if (r % 2) __builtin_amdgcn_sched_barrier(0);
  }
}
// The empty asm keeps each behind its (wave-uniform) branch: as selects, the compiler has every tile pay for them.
template <int AT, typename Hide>
__device__ __forceinline__ void mask_edge(const WinArgs& a, const Walk& w, const Edge& e, int t, Hide hide) {
  const bool back = behind<AT>(e);
  if (back && e.sinks > e.at + AT) {
    asm volatile("");
    mask_all<AT>(limits(a, w, e, t), hide);
    return;
  }
  if (back) {
    asm volatile("");
    mask_behind<AT>(limits(a, w, e, t).low, hide);
  }
  if (ahead<AT>(e)) {
    asm volatile("");
    mask_ahead<AT>(limits(a, w, e, t).up, hide);
  }
}

// The tiles, from the first up to but not including the second, of which all of a wave's tokens see all as far as the window goes: most of a long
// walk, where nothing else is looked at.
struct Span { int first, end; };
template <int T>
__device__ __forceinline__ Span whole_tiles(const WinArgs& a, const Walk& w, int first, int last) {
  const int left = last + w.shift - a.window, right = first + w.shift + 1;     // keys up to `left` are behind a token, from `right` on ahead of one
  return {uniform(w.sink_tiles + (left < 0 ? 0 : left / T + 1)), uniform(w.sink_tiles + (right < 0 ? 0 : right / T))};
}
// One load of 64 lanes: 16 bytes each from base + off to LDS at lds + AT.
template <int AT>
__device__ __forceinline__ void load_at(const uint16_t* base, unsigned off, int lds) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds), "n"(AT) : "memory", "m0", "scc");
}
// N of them, OFFS lane offsets: one for each, or one for all, whose bases are `step` elements apart.  (More than that are spilled in some kernels, and the
// wait for what was spilled is one for all loads on the way: backward of heads of 64 20 % slower.)
template <int N, int OFFS, int TO, int I = 0>
__device__ __forceinline__ void load_all(const uint16_t* base, int64_t step, const unsigned (&off)[OFFS], int lds) {
  load_at<I * TO>(base, off[OFFS == 1 ? 0 : I], lds);
  if constexpr (I + 1 < N) load_all<N, OFFS, TO, I + 1>(OFFS == 1 ? base + step : base, step, off, lds);
}
// Tiles of keys and values.  Whole ones whose rows are neighbours - all but the last of a range, a ring's end and few sinks - take lane offsets that are
// formed once.
template <int DH, int NW, int ROWS>
struct KeyLoads {
  typedef TileLoads<DH, NW, ROWS> Base;
  static constexpr int N = Base::N, OFFS = Base::kOneColumn ? 1 : N, PER_TILE = 2 * N;
  Base loads;
  const uint16_t* K; const uint16_t* V;                // the sequence's row 0
  unsigned off_k[OFFS], off_v[OFFS];
  __device__ __forceinline__ KeyLoads(const WinArgs& a, const Where& w, int wave) : loads(wave) {
    K = a.k + (int64_t)w.b * a.Sk * a.ldk + w.h * DH;
    V = a.v + (int64_t)w.b * a.Sk * a.ldv + w.h * DH;
#pragma unroll
    for (int i = 0; i < OFFS; ++i) {
      const unsigned r = loads.row + i * Base::STEP, c = loads.column(i) * 2;
      off_k[i] = r * (unsigned)(a.ldk * 2) + c;
      off_v[i] = r * (unsigned)(a.ldv * 2) + c;
      asm volatile("" : "+v"(off_k[i]), "+v"(off_v[i]));   // (of 64-bit products the low halves: else both are kept)
    }
  }
  // rows of the tile out of the ring's end, and repeats of the last one
  __device__ __forceinline__ void pieces(const WinArgs& a, const uint16_t* base, int64_t ld, const Tile& t, int m0v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r = loads.row + i * Base::STEP;
      r = t.row + (r < t.keys ? r : t.keys - 1);
      if (r >= a.Sk) r -= a.ring;
      const uint16_t* from = base + (int64_t)r * ld + loads.column(i);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(m0v + i * NW * 1024) : "memory", "m0");
    }
  }
  __device__ __forceinline__ void issue(const WinArgs& a, const Walk& w, int i, char* lds) const {
    const Tile t = tile_of<ROWS>(a, w, i);
    const int m0v = __builtin_amdgcn_readfirstlane((int)(size_t)lds + loads.wave * 1024);
    if (t.keys == ROWS && t.row + ROWS <= a.Sk) {
      load_all<N, OFFS, NW * 1024>(K + (int64_t)t.row * a.ldk, Base::STEP * a.ldk, off_k, m0v);
      load_all<N, OFFS, NW * 1024>(V + (int64_t)t.row * a.ldv, Base::STEP * a.ldv, off_v, m0v + ROWS * DH * 2);
    } else {
      pieces(a, K, a.ldk, t, m0v);
      pieces(a, V, a.ldv, t, m0v + ROWS * DH * 2);
    }
  }
};

// acc[dt] += tile^T p over SUBS x 32 streamed rows, which begin at lds
template <int DH, int SUBS>
__device__ __forceinline__ void add_product(f32x16 (&acc)[DH / 32], const char* lds, const Frag (&p)[SUBS][2]) {
#pragma unroll
  for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(lds, sub * 32 + ks * 16, dt * 32), p[sub][ks], acc[dt], 0, 0, 0);
}

// What a lane does not see has a probability of zero, and zero times an infinity or a NaN is none.  A wave whose sums are not finite forms them again,
// streamed row by streamed row in fp32 vector arithmetic out of global memory, leaving out for each lane what it does not see: many times slower,
// and with few registers, which the plain walk would else not have.
template <int N>
__device__ __forceinline__ bool finite(const f32x16 (&v)[N]) {
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = __fmaf_rn(v[i][r], 0.f, z);
  return z == 0.f;
}
template <int N>
__device__ __forceinline__ bool all_finite(const f32x16 (&v)[N]) { return __builtin_amdgcn_ballot_w64(!finite(v)) == 0; }
// a lane's own row times one that all share
template <int DH>
__device__ __forceinline__ float dot_row(const Frag (&own)[DH / 16], const uint16_t* row) {
  const int grp = (threadIdx.x & 63) >> 5;
  float s = 0.f;
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) {
    f32x4 x[2], y[2];
    bf16x8_to_f32(x, __builtin_bit_cast(u32x4, own[kk]));
    bf16x8_to_f32(y, *reinterpret_cast<const u32x4*>(row + kk * 16 + grp * 8));
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __fmaf_rn(x[e >> 2][e & 3], y[e >> 2][e & 3], s);
    __builtin_amdgcn_sched_barrier(0);
  }
  return s + __shfl_xor(s, 32, 64);
}
// acc += w row
template <int DH>
__device__ __forceinline__ void add_row(f32x16 (&acc)[DH / 32], float w, const uint16_t* row) {
  const int grp = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(row + dt * 32 + 8 * rg + 4 * grp);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[dt][4 * rg + e] = __fmaf_rn(w, __uint_as_float(e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16), acc[dt][4 * rg + e]);
      __builtin_amdgcn_sched_barrier(0);
    }
}
// every key of tiles t0, t0 + step .. of a walk with what a lane sees of it: use(row of the key, whether seen)
template <int T, typename Use>
__device__ __forceinline__ void one_by_one(const WinArgs& a, const Walk& w, int t0, int t1, int step, int t, int first, int last, Use use) {
  const int grp4 = (threadIdx.x & 32) >> 3;
#pragma unroll 1
  for (int i = t0; i < t1; i += step) {
    const Tile tile = tile_of<T>(a, w, i);
    const Limits v = limits(a, w, edge_of<T>(a, w, i, 0, first, last), t);
#pragma unroll 1
    for (int x = 0; x < tile.keys; ++x) use(tile.row + x < a.Sk ? tile.row + x : tile.row + x - a.ring, sees(v, x - grp4));
  }
}

// the larger of a lane's and of the lane 32 further on or back: a vector instruction, where __shfl_xor goes through LDS
__device__ __forceinline__ float other_half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// what scores of maximum m are formed from: of all -inf, as a part of a row's keys may be, 0, so that their probabilities are zero
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// Softmax of a tile of scores: s becomes exp2(s c2 - m), o is what was summed before.  m follows a row's maximum where that is kStay
// ahead of it: up to 2^8 in place of 1 loses nothing, and most tiles have a new maximum for one of a wave's 32 rows, which had all its sums multiplied.
constexpr float kStay = 8.0f;
template <int SUBS, int N>
__device__ __forceinline__ void softmax_tile(f32x16 (&s)[SUBS], const WinArgs& a, const Walk& w, bool whole, const Edge& e, int t, float& m, float& lsum, f32x16 (&o)[N]) {
  const float c2 = a.c2;
  if (!whole) {
    mask_edge<0>(a, w, e, t, [&](int r) { s[0][r] = -INFINITY; });
    if constexpr (SUBS == 2) mask_edge<32>(a, w, e, t, [&](int r) { s[SUBS - 1][r] = -INFINITY; });
  }
  float mx = s[0][0];
#pragma unroll
  for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[sub][r]);
  mx = other_half_max(mx);
  const bool ahead_of = mx * c2 > m + kStay;
  if (__builtin_amdgcn_ballot_w64(ahead_of)) {
    const float alpha = ahead_of ? __builtin_amdgcn_exp2f(m - mx * c2) : 1.0f;
    if (ahead_of) m = mx * c2;
    lsum *= alpha;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] *= alpha;
  }
  const float base = base_of(m);
  float ps = 0.f;
#pragma unroll
  for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[sub][r], c2, -base));
      s[sub][r] = p;
      ps += p;
    }
  lsum += ps;
}
// what a live row's sums end with: keys whose scores are all -inf have no softmax
__device__ __forceinline__ float log2_sum(float m, float tot) { return tot == 0.f ? NAN : m + __builtin_amdgcn_logf(tot); }

// ---- forward ----------------------------------------------------------------------------------
// A workgroup's own rows: tokens of one (sequence, key/value head), a wave's 32 of them and a lane's one.
template <int NW>
struct Rows {
  int start, n, live;                    // position of the sequence's first token, its tokens, their rows
  int r0, r, t, first, last;             // the workgroup's first row; a lane's row and token (of the last live row behind it); a wave's tokens
  bool active, gone;                     // whether a wave has live rows; whether a lane's row sees nothing
  __device__ __forceinline__ Rows(const WinArgs& a, const Where& w, int block, int wave) {
    start = start_of(a, w.b); n = live_of(a, w.b); live = n * a.share;
    r0 = block * OWN * NW;
    const int rw = r0 + wave * OWN;
    r = rw + (threadIdx.x & 31);
    active = rw < live;
    t = (r < live ? r : live > 0 ? live - 1 : 0) / a.share;
    first = __builtin_amdgcn_readfirstlane(t);
    last = __builtin_amdgcn_readlane(t, 31);
    gone = r >= live || (a.sinks == 0 && t < n - a.ring);        // padding; a token whose own key's row has been taken
  }
  template <int T>
  __device__ __forceinline__ Walk walk(const WinArgs& a) const {
    if (r0 >= live) return Walk{};
    const int end = r0 + OWN * NW < live ? r0 + OWN * NW : live;
    return walk_of<T>(a, start, n, r0 / a.share, (end - 1) / a.share);
  }
  __device__ __forceinline__ int clamped(int r_) const { return r_ < live ? r_ : live > 0 ? live - 1 : 0; }
};

template <int DH, int NW, int NS, int SUBS>
__global__ __launch_bounds__(64 * NW, NW / 4) void window_fwd_kernel(WinArgs a) {
  char* smem = dtl_smem;
  constexpr int SLOT = 2 * kTileBytes<DH>;               // keys, values
  const int parts = a.fwd.parts;
  Where w;
  if (!where(a, a.fwd, blockIdx.x, gridDim.x, w)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const Rows<NW> own(a, w, a.fwd.blocks - 1 - w.block, wave);    // later rows see more keys: they come first
  const Walk walk = own.template walk<TILE>(a);
  const int t0 = (int)((int64_t)walk.tiles * w.part / parts), t1 = (int)((int64_t)walk.tiles * (w.part + 1) / parts);
  const KeyLoads<DH, NW, TILE> loads(a, w, wave);
  const Span span = whole_tiles<TILE>(a, walk, own.first, own.last);
  constexpr int LPT = loads.PER_TILE;
  auto issue = [&](int i) { loads.issue(a, walk, i, smem + (i - t0) % NS * SLOT); };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (t0 + i < t1) issue(t0 + i);
  Frag qf[DH / 16];
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, own.clamped(own.r), a.ldq));
  settle(qf);
  f32x16 o[DH / 32];
  clear(o);
  float m = -INFINITY, lsum = 0.f;
  // SUBS x 32 keys of a tile
  auto some = [&](const char* Ks, bool whole, const Edge& e) {
    const char* Vs = Ks + kTileBytes<DH>;
    f32x16 s[SUBS];
    clear(s);
    in_a_row<SUBS * DH / 16, DH == 128 ? 6 : 3>([&](int i) { return frag_rows<DH>(Ks, i % SUBS * 32, i / SUBS); },
                        [&](int i, const Frag& f) { s[i % SUBS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i / SUBS], s[i % SUBS], 0, 0, 0); });
    softmax_tile(s, a, walk, whole, e, own.t, m, lsum, o);
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const Frag p[1][2] = {{pack_frag(s[sub], 0), pack_frag(s[sub], 1)}};
      add_product<DH, 1>(o, Vs + sub * 32 * DH * 2, p);
    }
  };
  auto tile = [&](int i, const char* Ks) {
#pragma unroll 1
    for (int at = 0; at < TILE; at += 32 * SUBS) {
      // (32 keys at a time the span costs more scalar registers than it saves comparisons: 4 x 2000 tokens of 16 heads, a window of 64 20.3 us, 19.3 without)
      const bool whole = SUBS == 2 && i >= span.first && i < span.end;
      Edge e{};
      if (!whole) e = edge_of<TILE>(a, walk, i, at, own.first, own.last);
      if (whole || !none<0>(e) || (SUBS == 2 && !none<32>(e))) some(Ks + at * DH * 2, whole, e);
    }
  };
  for (int i = t0; i < t1; ++i) {
    if (i + NS - 2 < t1) wait_loads<LPT * (NS - 2)>();
    else wait_loads<0>();
    __syncthreads();                                     // tile i is there, and everyone has left tile i - 1
    if (i + NS - 1 < t1) issue(i + NS - 1);
    if (own.active) tile(i, smem + (i - t0) % NS * SLOT);
  }
  if (own.active && !all_finite(o)) {
    clear(o);
    one_by_one<TILE>(a, walk, t0, t1, 1, own.t, own.first, own.last, [&](int row, bool seen) {
      const float s = dot_row<DH>(qf, loads.K + (int64_t)row * a.ldk);
      if (seen) add_row<DH>(o, __builtin_amdgcn_exp2f(__fmaf_rn(s, a.c2, -base_of(m))), loads.V + (int64_t)row * a.ldv);
    });
  }
  if (own.r >= a.R) return;
  const float tot = lsum + __shfl_xor(lsum, 32, 64);
  if (parts == 1) {
    if (own.gone) clear(o);
    store_owned<DH>(o, own.gone ? 0.f : 1.0f / tot, a.out + row_at<DH>(a, w.b, w.h, own.r, a.ldo));
    if (grp == 0) a.lse2[lse_at(a, w.b, w.h, own.r)] = own.gone ? -INFINITY : log2_sum(m, tot);
  } else if (!own.gone) {
    const int64_t at = ((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + own.r;
    store_owned32<DH>(o, a.part + at * DH);
    if (grp == 0) a.part_ml[at] = float2{m, tot};
  }
}

// Up to 32 rows to a key/value head - single tokens: bound by reading the keys and values once.  Each of the waves walks over tiles of 32 keys of its
// own, with a ring of its own and no barrier; their sums meet in LDS at the end.
constexpr int TOKEN_KEYS = 32;
constexpr int kTokenSlots = 2;
template <int DH> constexpr int kTokenRing = kTokenSlots * 2 * TOKEN_KEYS * DH * 2;   // of a wave
template <int DH, int TOKEN_NW>
__global__ __launch_bounds__(64 * TOKEN_NW) void window_token_kernel(WinArgs a) {
  constexpr int NS = kTokenSlots, HALF = TOKEN_KEYS * DH * 2, SLOT = 2 * HALF;
  const int parts = a.fwd.parts;
  Where w;
  if (!where(a, a.fwd, blockIdx.x, gridDim.x, w)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const Rows<1> own(a, w, 0, 0);
  const Walk walk = own.template walk<TOKEN_KEYS>(a);
  const int t0 = (int)((int64_t)walk.tiles * w.part / parts), t1 = (int)((int64_t)walk.tiles * (w.part + 1) / parts);
  char* ring = dtl_smem + wave * kTokenRing<DH>;
  const KeyLoads<DH, 1, TOKEN_KEYS> loads(a, w, 0);
  constexpr int LPT = loads.PER_TILE;
  const int mine = t1 - t0 > wave ? (t1 - t0 - wave + TOKEN_NW - 1) / TOKEN_NW : 0;      // tiles t0 + wave, + TOKEN_NW, ...
  auto issue = [&](int i) { loads.issue(a, walk, t0 + wave + i * TOKEN_NW, ring + i % NS * SLOT); };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < mine) issue(i);
  Frag qf[DH / 16];
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, own.clamped(own.r), a.ldq));
  settle(qf);
  f32x16 o[DH / 32];
  clear(o);
  float m = -INFINITY, lsum = 0.f;
  for (int i = 0; i < mine; ++i) {
    // the slot that is filled next was read a tile ago; its reads have come back before the load goes out
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    if (i + NS - 1 < mine) { issue(i + NS - 1); wait_loads<LPT * (NS - 1)>(); }
    else wait_loads<0>();
    const char* Ks = ring + i % NS * SLOT;
    const Edge e = edge_of<TOKEN_KEYS>(a, walk, t0 + wave + i * TOKEN_NW, 0, own.first, own.last);
    f32x16 s[1];
    clear(s);
    in_a_row<DH / 16, 4>([&](int i) { return frag_rows<DH>(Ks, 0, i); },
                         [&](int i, const Frag& f) { s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i], s[0], 0, 0, 0); });
    softmax_tile(s, a, walk, false, e, own.t, m, lsum, o);
    const Frag p[1][2] = {{pack_frag(s[0], 0), pack_frag(s[0], 1)}};
    add_product<DH, 1>(o, Ks + HALF, p);
  }
  if (own.first != own.last && !all_finite(o)) {         // (one token: what is masked is a repeat of what it sees)
    clear(o);
    one_by_one<TOKEN_KEYS>(a, walk, t0 + wave, t1, TOKEN_NW, own.t, own.first, own.last, [&](int row, bool seen) {
      const float s = dot_row<DH>(qf, loads.K + (int64_t)row * a.ldk);
      if (seen) add_row<DH>(o, __builtin_amdgcn_exp2f(__fmaf_rn(s, a.c2, -base_of(m))), loads.V + (int64_t)row * a.ldv);
    });
  }
  lsum += __shfl_xor(lsum, 32, 64);
  // the waves' sums: registers through LDS, an equal share of them to each wave
  __syncthreads();
  float* image = reinterpret_cast<float*>(dtl_smem);     // [wave][DH / 2][64], then the pairs
  float2* ml = reinterpret_cast<float2*>(image + TOKEN_NW * (DH / 2) * 64);
  const int r = l & 31;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) image[(wave * (DH / 2) + dt * 16 + x) * 64 + l] = o[dt][x];
  if (grp == 0) ml[wave * 32 + r] = float2{m, lsum};
  __syncthreads();
  float top = -INFINITY, tot = 0.f, f[TOKEN_NW];
#pragma unroll
  for (int i = 0; i < TOKEN_NW; ++i) top = fmaxf(top, ml[i * 32 + r].x);
  const float base = base_of(top);
#pragma unroll
  for (int i = 0; i < TOKEN_NW; ++i) {
    f[i] = __builtin_amdgcn_exp2f(ml[i * 32 + r].x - base);
    tot += ml[i * 32 + r].y * f[i];
  }
  if (r >= a.R || (parts > 1 && own.gone)) return;
  const int64_t at = ((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + r;
  const float inv = 1.0f / tot;
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
    if (parts > 1) { *reinterpret_cast<f32x4*>(a.part + at * DH + col) = v; continue; }
    v *= inv;
    if (own.gone) v = f32x4{0.f, 0.f, 0.f, 0.f};
    *reinterpret_cast<u32x2*>(out + col) = u32x2{rv_pack_bf16x2(v.x, v.y), rv_pack_bf16x2(v.z, v.w)};
  }
  if (wave != 0 || grp != 0) return;
  if (parts > 1) a.part_ml[at] = float2{top, tot};
  else a.lse2[lse_at(a, w.b, w.h, r)] = own.gone ? -INFINITY : log2_sum(top, tot);
}

// parts -> out, lse2.  Eight columns to a lane; LANES lanes share the parts of one.
template <int DH, int LANES>
__global__ __launch_bounds__(256) void window_join_kernel(WinArgs a) {
  constexpr int W = 256 / LANES;                         // column groups of a block
  static_assert(W % (DH / 8) == 0, "whole rows");
  __shared__ f32x4 sums[2][256];
  __shared__ float2 pairs[256];
  const int64_t rows = (int64_t)a.B * a.Hkv * a.R;
  const int lane = threadIdx.x / W;
  const int64_t i = (int64_t)blockIdx.x * W + threadIdx.x % W, row = i / (DH / 8);
  const int c = (int)(i % (DH / 8)) * 8;
  const int unit = row < rows ? (int)(row / a.R) : 0, r = (int)(row - (int64_t)unit * a.R);
  bool gone = true;
  if (row < rows) {
    const int n = live_at(a, unit / a.Hkv), t = r / a.share;
    gone = t >= n || (a.sinks == 0 && t < n - a.ring);
  }
  float m = -INFINITY, tot = 0.f;
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  auto add = [&](float2 ml, f32x4 x, f32x4 y) {
    const float mn = fmaxf(m, ml.x), base = base_of(mn);
    const float was = __builtin_amdgcn_exp2f(m - base), f = __builtin_amdgcn_exp2f(ml.x - base);
    v[0] = v[0] * was + x * f;
    v[1] = v[1] * was + y * f;
    tot = tot * was + ml.y * f;
    m = mn;
  };
  if (!gone) {
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
  const float inv = gone ? 0.f : 1.0f / tot;
  v[0] *= inv; v[1] *= inv;
  *reinterpret_cast<u32x4*>(a.out + row_at<DH>(a, unit / a.Hkv, unit % a.Hkv, r, a.ldo) + c) = f32_to_bf16x8(v);
  if (c == 0) a.lse2[lse_at(a, unit / a.Hkv, unit % a.Hkv, r)] = gone ? -INFINITY : log2_sum(m, tot);
}

// ---- backward (of a call without a cache: keys are the tokens' own) ---------------------------------
// What the accumulators of the scores and of do v^T begin with, for every row in the order of the list: -lse / c2, so that a probability is
// exp2(c2 acc), and -D = -rowsum(do o), so that acc is dp - D.  Behind the last row and for padding -inf, which makes the
// probabilities zero, and 0.
template <int DH>
__global__ __launch_bounds__(256) void window_stat_kernel(WinArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / (DH / 8);
  const int c = (int)(i % (DH / 8)) * 8;
  if (row >= (int64_t)a.B * a.Hkv * a.Rp) return;         // (whole rows: DH / 8 lanes go together)
  const int unit = (int)(row / a.Rp), r = (int)(row - (int64_t)unit * a.Rp);
  const int b = unit / a.Hkv, h = unit % a.Hkv;
  float d = 0.f, lse = INFINITY;
  if (r < live_at(a, b) * a.share) {
    f32x4 x[2], y[2];
    bf16x8_to_f32(x, *reinterpret_cast<const u32x4*>(a.o + row_at<DH>(a, b, h, r, a.ldo) + c));
    bf16x8_to_f32(y, *reinterpret_cast<const u32x4*>(a.dout + row_at<DH>(a, b, h, r, a.lddo) + c));
#pragma unroll
    for (int k = 0; k < 8; ++k) d = __fmaf_rn(x[k >> 2][k & 3], y[k >> 2][k & 3], d);
    lse = a.lse2[lse_at(a, b, h, r)];
    lse = lse == -INFINITY ? INFINITY : lse / a.c2;
  }
#pragma unroll
  for (int o = 1; o < DH / 8; o *= 2) d += __shfl_xor(d, o, 64);
  if (c == 0) { a.stat_lse[row] = -lse; a.stat_d[row] = lse == INFINITY ? 0.f : -d; }
}

// every token sees but one key: its score's gradient is zero
__device__ __forceinline__ bool one_key(const WinArgs& a, int n) { return n == 1 || (a.window == 1 && a.sinks == 0); }

// dQ: a wave owns 32 rows, keys and values stream.
template <int DH, int NW, int NS>
__device__ __forceinline__ void bwd_q_body(const WinArgs& a, int id, int grid) {
  char* smem = dtl_smem;
  constexpr int SLOT = 2 * kTileBytes<DH>;
  const int parts = a.bq.parts;
  Where w;
  if (!where(a, a.bq, id, grid, w)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const Rows<NW> own(a, w, a.bq.blocks - 1 - w.block, wave);
  const Walk walk = own.template walk<TILE>(a);
  const int t0 = (int)((int64_t)walk.tiles * w.part / parts), t1 = (int)((int64_t)walk.tiles * (w.part + 1) / parts);
  f32x16 dq[DH / 32];
  clear(dq);
  const KeyLoads<DH, NW, TILE> loads(a, w, wave);
  constexpr int LPT = loads.PER_TILE;
  auto issue = [&](int i) { loads.issue(a, walk, i, smem + (i - t0) % NS * SLOT); };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (t0 + i < t1) issue(t0 + i);
  Frag qf[DH / 16], of[DH / 16];
  const int rc = own.clamped(own.r);
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, rc, a.ldq));
  load_owned<DH>(of, a.dout + row_at<DH>(a, w.b, w.h, rc, a.lddo));
  float lse = a.stat_lse[(int64_t)w.unit * a.Rp + rc], D = a.stat_d[(int64_t)w.unit * a.Rp + rc];
  settle(qf); settle(of);
  asm volatile("" : "+v"(lse), "+v"(D));
  auto tile = [&](int i, const char* Ks) {
    const char* Vs = Ks + kTileBytes<DH>;
#pragma unroll(DH == 128 ? 1 : 2)
    for (int sub = 0; sub < 2; ++sub) {
      const Edge e = edge_of<TILE>(a, walk, i, sub * 32, own.first, own.last);
      if (none<0>(e)) continue;
      f32x16 s[1], dp[1];
#pragma unroll
      for (int x = 0; x < 16; ++x) { s[0][x] = lse; dp[0][x] = D; }
      in_a_row<DH / 8, DH == 128 ? 4 : 2>([&](int i) { return frag_rows<DH>(i % 2 ? Vs : Ks, sub * 32, i / 2); },
                          [&](int i, const Frag& f) {
                            if (i % 2) dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, of[i / 2], dp[0], 0, 0, 0);
                            else s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i / 2], s[0], 0, 0, 0);
                          });
#pragma unroll
      for (int x = 0; x < 16; ++x) dp[0][x] *= __builtin_amdgcn_exp2f(s[0][x] * a.c2);
      mask_edge<0>(a, walk, e, own.t, [&](int r) { dp[0][r] = 0.f; });
      const Frag ds[1][2] = {{pack_frag(dp[0], 0), pack_frag(dp[0], 1)}};
      add_product<DH, 1>(dq, Ks + sub * 32 * DH * 2, ds);
    }
  };
  for (int i = t0; i < t1; ++i) {
    if (i + NS - 2 < t1) wait_loads<LPT * (NS - 2)>();
    else wait_loads<0>();
    __syncthreads();
    if (i + NS - 1 < t1) issue(i + NS - 1);
    if (own.active) tile(i, smem + (i - t0) % NS * SLOT);
  }
  if (own.active && !all_finite(dq)) {
    clear(dq);
    one_by_one<TILE>(a, walk, t0, t1, 1, own.t, own.first, own.last, [&](int row, bool seen) {
      const uint16_t* k = loads.K + (int64_t)row * a.ldk;
      const float p = __builtin_amdgcn_exp2f((lse + dot_row<DH>(qf, k)) * a.c2), dp = D + dot_row<DH>(of, loads.V + (int64_t)row * a.ldv);
      if (seen) add_row<DH>(dq, p * dp, k);
    });
  }
  if (own.r >= a.R) return;
  if (own.gone) clear(dq);
  else if (one_key(a, own.n)) of_one_key(dq);
  if (parts == 1) store_owned<DH>(dq, a.scale, a.dq + row_at<DH>(a, w.b, w.h, own.r, a.lddq));
  else store_owned32<DH>(dq, a.q_part + (((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + own.r) * DH);
}

// Tiles of rows: queries and do.  Where a load's rows are whole tokens, lane offsets are formed once.
template <int DH, int NW, int ROWS>
struct RowLoads {
  typedef TileLoads<DH, NW, ROWS> Base;
  static constexpr int N = Base::N;
  Base loads;
  int tokens;                                          // of a load's step, or 0
  unsigned off_q[1], off_o[1];
  __device__ __forceinline__ RowLoads(const WinArgs& a, int wave) : loads(wave) {
    tokens = Base::kOneColumn && Base::STEP % a.share == 0 ? Base::STEP / a.share : 0;
    const unsigned t = loads.row / a.share, c = ((loads.row - t * a.share) * DH + loads.column(0)) * 2;
    off_q[0] = t * (unsigned)(a.ldq * 2) + c;
    off_o[0] = t * (unsigned)(a.lddo * 2) + c;
    asm volatile("" : "+v"(off_q[0]), "+v"(off_o[0]));
  }
  // tile i of the rows of (b, h) from token t0 on, no further than row `end`
  __device__ __forceinline__ void issue(const WinArgs& a, int b, int h, int t0, int i, int end, char* lds) const {
    const int r0 = t0 * a.share + i * ROWS;
    if (tokens && r0 + ROWS <= end) {
      const int64_t tok = (int64_t)b * a.Sq + t0 + i * N * tokens;
      const int m0v = __builtin_amdgcn_readfirstlane((int)(size_t)lds + loads.wave * 1024);
      load_all<N, 1, NW * 1024>(a.q + tok * a.ldq + h * a.share * DH, tokens * a.ldq, off_q, m0v);
      load_all<N, 1, NW * 1024>(a.dout + tok * a.lddo + h * a.share * DH, tokens * a.lddo, off_o, m0v + ROWS * DH * 2);
      return;
    }
    loads.rows([&](int r, int64_t& tok, int& c) {
      const int t = r / a.share, g = r - t * a.share;
      tok = (int64_t)b * a.Sq + t;
      c = (h * a.share + g) * DH;
    }, end, a.q, a.ldq, a.dout, a.lddo, r0, lds, lds + ROWS * DH * 2);
  }
};

// dK, dV of the window: a wave owns 32 keys, the rows (queries and do) of the tokens whose windows hold any of a workgroup's keys stream.
template <int DH, int NW, int NS, int ROWS>
__device__ __forceinline__ void bwd_kv_body(const WinArgs& a, int id, int grid) {
  char* smem = dtl_smem;
  constexpr int HALF = ROWS * DH * 2, SLOT = 2 * HALF + 2 * 64 * 4;   // queries, do, lse, D
  const int parts = a.bkv.parts;
  Where w;
  if (!where(a, a.bkv, id, grid, w)) return;
  const int n = live_of(a, w.b), j0 = w.block * OWN * NW;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const int j = j0 + wave * OWN + (l & 31);
  // rows whose window holds key x: x share .. end(x) - 1
  auto end = [&](int x) { return (n - x < a.window ? n : x + a.window) * a.share; };
  const int jl = (j0 + OWN * NW < n ? j0 + OWN * NW : n) - 1;                 // the workgroup's last key
  const int from = j0 * a.share, to_row = j0 < n ? end(jl) : from;
  const int nt = (to_row - from + ROWS - 1) / ROWS;         // keys behind the sequence: zeros
  const int t0 = (int)((int64_t)nt * w.part / parts), t1 = (int)((int64_t)nt * (w.part + 1) / parts);
  const bool active = j0 + wave * OWN < n;
  const int jc = j < n ? j : n > 0 ? n - 1 : 0, w0 = __builtin_amdgcn_readfirstlane(jc), w1 = __builtin_amdgcn_readlane(jc, 31);
  const int my_first = jc * a.share, my_end = end(jc);
  const int all_first = w1 * a.share, all_end = end(w0), any_first = w0 * a.share, any_end = end(w1);
  // Keys, values, their two gradients and the scores are 256 registers by themselves (heads of 64: 144 of 168): the values stay in LDS
  Frag* vl = reinterpret_cast<Frag*>(smem + NS * SLOT + wave * OWN * DH * 2) + l;
  Frag kf[DH / 16], vf[DH / 16];
  f32x16 dk[DH / 32], dv[DH / 32];
  clear(dk); clear(dv);
  const RowLoads<DH, NW, ROWS> loads(a, wave);
  constexpr int LPT = 2 * RowLoads<DH, NW, ROWS>::N + 1;
  const float* stat = (wave & 1 ? a.stat_d : a.stat_lse) + (int64_t)w.unit * a.Rp;   // (even waves bring the lse, odd ones D)
  auto issue = [&](int i) {
    char* to = smem + (i - t0) % NS * SLOT;
    loads.issue(a, w.b, w.h, j0, i, to_row, to);
    load_floats(stat + from + i * ROWS, to + 2 * HALF + (wave & 1) * 64 * 4);
  };
  // The first tiles go out ahead of the wave's own keys: with few rows a workgroup is one chain of round trips.
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (t0 + i < t1) issue(t0 + i);
  if (active) {
    load_owned<DH>(kf, a.k + ((int64_t)w.b * a.Sk + jc) * a.ldk + w.h * DH);
    load_owned<DH>(vf, a.v + ((int64_t)w.b * a.Sk + jc) * a.ldv + w.h * DH);
    settle(kf); settle(vf);
#pragma unroll
    for (int kk = 0; kk < DH / 16; ++kk) vl[kk * 64] = vf[kk];
  }
  auto tile = [&](int i, const char* Qs) {
    const char* Os = Qs + HALF;
    const float* lse = reinterpret_cast<const float*>(Os + HALF);
#pragma unroll(DH == 128 ? 1 : 2)
    for (int sub = 0; sub < ROWS / 32; ++sub) {
      const int r0 = from + i * ROWS + sub * 32;
      if (r0 + 31 < any_first || r0 >= any_end) continue;
      f32x16 s[1], dp[1];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 ls = *reinterpret_cast<const f32x4*>(lse + sub * 32 + 8 * q + 4 * grp);
        const f32x4 D = *reinterpret_cast<const f32x4*>(lse + 64 + sub * 32 + 8 * q + 4 * grp);
#pragma unroll
        for (int x = 0; x < 4; ++x) { s[0][4 * q + x] = ls[x]; dp[0][4 * q + x] = D[x]; }
      }
      struct Two { Frag rows, values; };
      in_a_row<DH / 8, DH == 128 ? 4 : 2>([&](int i) {
                            Two t;
                            t.rows = frag_rows<DH>(i % 2 ? Os : Qs, sub * 32, i / 2);
                            if (i % 2) t.values = vl[i / 2 * 64];
                            return t;
                          },
                          [&](int i, const Two& t) {
                            if (i % 2) dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, t.values, dp[0], 0, 0, 0);
                            else s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, kf[i / 2], s[0], 0, 0, 0);
                          });
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[0][x] = __builtin_amdgcn_exp2f(s[0][x] * a.c2);
        dp[0][x] *= s[0][x];
      }
      auto hide = [&](int r) { s[0][r] = dp[0][r] = 0.f; };
      if (r0 < all_first) {                                // (wave-uniform)
        asm volatile("");
        mask_behind<0>(my_first - 1 - r0 - 4 * grp, hide);
      }
      if (r0 + 32 > all_end) {
        asm volatile("");
        mask_ahead<0>(my_end - 1 - r0 - 4 * grp, hide);
      }
      const Frag p[1][2] = {{pack_frag(s[0], 0), pack_frag(s[0], 1)}}, ds[1][2] = {{pack_frag(dp[0], 0), pack_frag(dp[0], 1)}};
      const char* O = Os + sub * 32 * DH * 2;
      const char* Q = Qs + sub * 32 * DH * 2;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt) {
          dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(O, ks * 16, dt * 32), p[0][ks], dv[dt], 0, 0, 0);
          dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Q, ks * 16, dt * 32), ds[0][ks], dk[dt], 0, 0, 0);
        }
    }
  };
  for (int i = t0; i < t1; ++i) {
    if (i + NS - 2 < t1) wait_loads<LPT * (NS - 2)>();
    else wait_loads<0>();
    __syncthreads();
    if (i + NS - 1 < t1) issue(i + NS - 1);
    if (active) tile(i, smem + (i - t0) % NS * SLOT);
  }
  if (active && !(all_finite(dk) && all_finite(dv))) {
    clear(dk); clear(dv);
    load_owned<DH>(vf, a.v + ((int64_t)w.b * a.Sk + jc) * a.ldv + w.h * DH);
    const int r1 = from + t1 * ROWS < to_row ? from + t1 * ROWS : to_row;
    const float* lse = a.stat_lse + (int64_t)w.unit * a.Rp;
    const float* D = a.stat_d + (int64_t)w.unit * a.Rp;
#pragma unroll 1
    for (int r = from + t0 * ROWS; r < r1; ++r) {
      const uint16_t* q = a.q + row_at<DH>(a, w.b, w.h, r, a.ldq);
      const uint16_t* d = a.dout + row_at<DH>(a, w.b, w.h, r, a.lddo);
      const float p = __builtin_amdgcn_exp2f((lse[r] + dot_row<DH>(kf, q)) * a.c2), dp = D[r] + dot_row<DH>(vf, d);
      if (r < my_first || r >= my_end) continue;
      add_row<DH>(dv, p, d);
      add_row<DH>(dk, p * dp, q);
    }
  }
  if (j >= a.Sk) return;
  if (one_key(a, n)) of_one_key(dk);
  if (j >= n) { clear(dk); clear(dv); }                     // (repeats of the last key)
  if (a.sink_parts && j < a.sinks) return;                  // bwd_sink_body's
  if (parts == 1) {
    store_owned<DH>(dk, a.scale, a.dk + ((int64_t)w.b * a.Sk + j) * a.lddk + w.h * DH);
    store_owned<DH>(dv, 1.0f, a.dv + ((int64_t)w.b * a.Sk + j) * a.lddv + w.h * DH);
  } else {
    float* to = a.kv_part + (((int64_t)w.part * a.B * a.Hkv + w.unit) * a.Sk + j) * 2 * DH;
    store_owned32<DH>(dk, to);
    store_owned32<DH>(dv, to + DH);
  }
}

// dK, dV of the sinks, which all rows behind them see: 32 keys, thousands of rows.  The four waves of a workgroup own the same keys and walk over 32 rows
// each in turn, in slots of their own and without barriers; their sums meet in LDS and are the result, or a part of it.
// (The first block of keys had all the rows at first, one workgroup's walk: 4 x 4096 tokens, 16 heads over 2 of 128, a window of 1024, 1568 us, 523 without.)
template <int DH>
__device__ __forceinline__ void bwd_sink_body(const WinArgs& a, int id) {
  constexpr int ROWS = 32, HALF = ROWS * DH * 2, SLOT = 2 * HALF;
  const int part = id % a.sink_parts, block = id / a.sink_parts % a.sink_blocks, unit = id / a.sink_parts / a.sink_blocks;
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const int n = live_of(a, b), j0 = block * OWN, j = j0 + (l & 31);
  const int last = a.sinks - 1 < n - 1 ? a.sinks - 1 : n - 1, jc = j < last ? j : last > 0 ? last : 0;
  const int from_token = j0 < n ? j0 : n, from = from_token * a.share, to_row = n * a.share;
  const int nt = (to_row - from + ROWS - 1) / ROWS;
  const int t0 = (int)((int64_t)nt * part / a.sink_parts), t1 = (int)((int64_t)nt * (part + 1) / a.sink_parts);
  const int my_first = jc * a.share, all_first = __builtin_amdgcn_readlane(my_first, 31);
  char* slot = dtl_smem + wave * SLOT;
  // keys and values in LDS, one copy for all waves: with both gradients and the scores they are too many registers
  Frag* own = reinterpret_cast<Frag*>(dtl_smem + 4 * SLOT) + l;
  const uint16_t* K = a.k + ((int64_t)b * a.Sk + jc) * a.ldk + h * DH;
  const uint16_t* V = a.v + ((int64_t)b * a.Sk + jc) * a.ldv + h * DH;
  if (wave < 2) {
    Frag f[DH / 16];
    load_owned<DH>(f, wave ? V : K);
#pragma unroll
    for (int kk = 0; kk < DH / 16; ++kk) own[(2 * kk + wave) * 64] = f[kk];
  }
  __syncthreads();
  f32x16 dk[DH / 32], dv[DH / 32];
  clear(dk); clear(dv);
  const RowLoads<DH, 1, ROWS> loads(a, 0);
  const float* stat_lse = a.stat_lse + (int64_t)unit * a.Rp;
  const float* stat_d = a.stat_d + (int64_t)unit * a.Rp;
  const int first = t0 + wave;
#pragma unroll 1
  for (int i = first; i < t1; i += 4) {
    const int r0 = from + i * ROWS;
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");      // the reads of the rows before have come back
    int same = 0;
    asm volatile("" : "+s"(same));                            // (fragments' addresses are not kept over the loop: there are no registers for them)
    char* Qs = slot + same;
    loads.issue(a, b, h, from_token, i, to_row, Qs);
    f32x16 s[1], dp[1];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[0][4 * q + x] = stat_lse[r0 + 8 * q + 4 * grp + x];
        dp[0][4 * q + x] = stat_d[r0 + 8 * q + 4 * grp + x];
      }
    wait_loads<0>();
    const char* Os = Qs + HALF;
    struct Two { Frag rows, own; };
#pragma unroll 1
    for (int k0 = 0; k0 < DH / 8; k0 += 8)                      // (all at once, the compiler reads all fragments before the first product)
      in_a_row<8, 2>([&](int i) {
                       Two t;
                       t.rows = frag_rows<DH>(i % 2 ? Os : Qs, 0, (k0 + i) / 2);
                       t.own = own[(k0 + i) * 64];
                       return t;
                     },
                     [&](int i, const Two& t) {
                       if (i % 2) dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, t.own, dp[0], 0, 0, 0);
                       else s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, t.own, s[0], 0, 0, 0);
                     });
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[0][x] = __builtin_amdgcn_exp2f(s[0][x] * a.c2);
      dp[0][x] *= s[0][x];
    }
    auto hide = [&](int r) { s[0][r] = dp[0][r] = 0.f; };
    if (r0 < all_first) {
      asm volatile("");
      mask_behind<0>(my_first - 1 - r0 - 4 * grp, hide);
    }
    if (r0 + ROWS > to_row) {
      asm volatile("");
      mask_ahead<0>(to_row - 1 - r0 - 4 * grp, hide);
    }
    const Frag p[1][2] = {{pack_frag(s[0], 0), pack_frag(s[0], 1)}}, ds[1][2] = {{pack_frag(dp[0], 0), pack_frag(dp[0], 1)}};
    add_product<DH, 1>(dv, Os, p);
    add_product<DH, 1>(dk, Qs, ds);
  }
  if (!(all_finite(dk) && all_finite(dv))) {
    clear(dk); clear(dv);
    Frag kf[DH / 16], vf[DH / 16];
    load_owned<DH>(kf, K);
    load_owned<DH>(vf, V);
#pragma unroll 1
    for (int i = first; i < t1; i += 4) {
      const int r1 = from + (i + 1) * ROWS < to_row ? from + (i + 1) * ROWS : to_row;
#pragma unroll 1
      for (int r = from + i * ROWS; r < r1; ++r) {
        const uint16_t* q = a.q + row_at<DH>(a, b, h, r, a.ldq);
        const uint16_t* d = a.dout + row_at<DH>(a, b, h, r, a.lddo);
        const float pr = __builtin_amdgcn_exp2f((stat_lse[r] + dot_row<DH>(kf, q)) * a.c2), dp = stat_d[r] + dot_row<DH>(vf, d);
        if (r < my_first) continue;
        add_row<DH>(dv, pr, d);
        add_row<DH>(dk, pr * dp, q);
      }
    }
  }
  if (n == 1) of_one_key(dk);
  if (j >= n) { clear(dk); clear(dv); }                       // (repeats of the last key)
  // the waves' sums, dk's and then dv's: registers through LDS, an equal share of them to each wave
  float* image = reinterpret_cast<float*>(dtl_smem);          // [4][DH / 2][64]: the slots
  float* to = a.sink_part + (((int64_t)part * a.B * a.Hkv + unit) * a.sinks + j) * 2 * DH;
#pragma unroll
  for (int what = 0; what < 2; ++what) {
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int x = 0; x < 16; ++x) image[(wave * (DH / 2) + dt * 16 + x) * 64 + l] = what ? dv[dt][x] : dk[dt][x];
    __syncthreads();
    if (j >= a.sinks) continue;
    uint16_t* out = what ? a.dv + ((int64_t)b * a.Sk + j) * a.lddv + h * DH : a.dk + ((int64_t)b * a.Sk + j) * a.lddk + h * DH;
    const float mul = what ? 1.0f : a.scale;
#pragma unroll
    for (int x = 0; x < DH / 8; x += 4) {
      const int reg = wave * (DH / 8) + x, col = (reg >> 4) * 32 + acc_row(reg & 15, grp);
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[e] += image[(i * (DH / 2) + reg + e) * 64 + l];
      }
      if (a.sink_parts > 1) *reinterpret_cast<f32x4*>(to + what * DH + col) = v;
      else *reinterpret_cast<u32x2*>(out + col) = u32x2{rv_pack_bf16x2(v.x * mul, v.y * mul), rv_pack_bf16x2(v.z * mul, v.w * mul)};
    }
  }
}
template <int DH> constexpr int kSinkLds = 4 * 2 * 32 * DH * 2 + 2 * 32 * DH * 2;
template <int DH, int NW, int NS, int ROWS> constexpr int kKvLds = NS * (2 * ROWS * DH * 2 + 2 * 64 * 4) + NW * OWN * DH * 2;
template <int DH, int NS> constexpr int kQLds = NS * 2 * kTileBytes<DH>;
constexpr int most(int x, int y) { return x > y ? x : y; }
template <int DH, int NW, int NS, int ROWS, int NS_Q> constexpr int kBwdLds = most(kKvLds<DH, NW, NS, ROWS>, most(kQLds<DH, NS_Q>, kSinkLds<DH>));
// All in one launch, the longer workgroups (dK and dV: four products to dQ's three) first.
template <int DH, int NW, int NS, int ROWS, int NS_Q>
__global__ __launch_bounds__(64 * NW, DH == 128 ? 2 : 3) void window_bwd_kernel(WinArgs a) {
  static_assert(NW == 4, "bwd_sink_body");
  const int id = blockIdx.x, others = a.kv_grid + a.sink_grid;
  if (id < a.kv_grid) bwd_kv_body<DH, NW, NS, ROWS>(a, id, a.kv_grid);
  else if (id < others) bwd_sink_body<DH>(a, id - a.kv_grid);
  else bwd_q_body<DH, NW, NS_Q>(a, id - others, gridDim.x - others);
}
// parts -> dq (KV false), or dk and dv, of the sinks alone where the others' are no parts
template <int DH, bool KV>
__global__ __launch_bounds__(256) void window_bwd_join_kernel(WinArgs a) {
  constexpr int W = KV ? 2 * DH : DH;
  const int per = !KV ? a.R : a.bkv.parts > 1 ? a.Sk : a.sinks;
  const int64_t units = (int64_t)a.B * a.Hkv, i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / (W / 8);
  const int c = (int)(i % (W / 8)) * 8;
  if (row >= units * per) return;
  const int unit = (int)(row / per), r = (int)(row - (int64_t)unit * per), b = unit / a.Hkv, h = unit % a.Hkv;
  const bool sink = KV && a.sink_parts && r < a.sinks;
  if (sink && a.sink_parts == 1) return;                    // there already
  const int parts = !KV ? a.bq.parts : sink ? a.sink_parts : a.bkv.parts, rows = !KV ? a.R : sink ? a.sinks : a.Sk;
  const float* from = (!KV ? a.q_part : sink ? a.sink_part : a.kv_part) + ((int64_t)unit * rows + r) * W + c;
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
  for (int s = 0; s < parts; ++s) {
    const f32x4* p = reinterpret_cast<const f32x4*>(from + s * units * rows * W);
    v[0] += p[0]; v[1] += p[1];
  }
  const bool values = KV && c >= DH;
  if (!values) { v[0] *= a.scale; v[1] *= a.scale; }
  uint16_t* to = !KV ? a.dq + row_at<DH>(a, b, h, r, a.lddq) + c
                 : values ? a.dv + ((int64_t)b * a.Sk + r) * a.lddv + h * DH + c - DH : a.dk + ((int64_t)b * a.Sk + r) * a.lddk + h * DH + c;
  *reinterpret_cast<u32x4*>(to) = f32_to_bf16x8(v);
}

// ---- host ----------------------------------------------------------------------------------
// Waves of a workgroup of single tokens: rings of 128 KB, one workgroup to a CU, or of 64 KB where there is more than one to each.  us, 128 / 64 KB: a
// token of 16 heads over 2 of 64 and 4000 keys, 4 sequences 18.2 / 37.9 (with the join's 4); 20 sequences of 8 heads of 128 and 2000 keys 32 / 40;
// 32 of 32 over 8 of 128 and 4100 keys 100 / 99, 5.4 TB/s; 20 of 8 heads of 64 and 32000 keys 303 / 294.
template <int DH, bool WIDE> constexpr int kTokenWaves = (DH == 128 ? 2 : 4) * (WIDE ? 2 : 1);
constexpr int64_t kTokenGrid = 256;

struct WinPlan {
  bool token, wide;                        // up to 32 rows to a key/value head; workgroups of more waves
  int R, Rp, fwd_parts, q_parts, kv_parts, sink_blocks, sink_parts;
  int window, sinks;                       // no more than the rows
  int at_once;                             // sequences
  size_t fwd_ml, fwd_bytes;                // forward: [sums][pairs]
  size_t d, part, kv_part, sink_part, bwd_bytes;   // backward: [lse][D][sums of dq][of dk and dv][of the sinks']
};
bool make_plan(WinPlan& p, int64_t B, int64_t Sq, int64_t Sk, int64_t H, int64_t Hkv, int64_t dh, int64_t window, int64_t sinks, bool backward) {
  if (B < 1 || Sq < 1 || Sk < 1 || H < 1 || Hkv < 1 || H % Hkv || (dh != 64 && dh != 128) || window < 1 || sinks < 0) return false;
  if (B > (1 << 20) || Sq > (1 << 24) || Sk > (1 << 24) || H > (1 << 16) || (backward && Sq != Sk)) return false;
  const int64_t U = B * Hkv, share = H / Hkv, R = share * Sq;
  if (R > (1ll << 30) - 64 || U * up(R, OWN) > (1ll << 30) || U * up(Sk, OWN) > (1ll << 30)) return false;
  if (U * R * dh / 8 > (1ll << 38) || U * Sk * dh / 8 > (1ll << 38)) return false;
  p.window = (int)(window < Sk ? window : Sk);
  p.sinks = (int)(sinks < Sk ? sinks : Sk - 1);
  p.R = (int)R; p.Rp = (int)(up(R + TILE - 1, TILE) * TILE);  // (a tile of rows may begin at any of them)
  p.token = R <= OWN;
  // tiles that a workgroup of `rows` walks over at most
  auto tiles = [&](int64_t rows, int64_t T) {
    int64_t span = p.window + (rows - 1) / share + 1;
    span = span < Sk ? span : Sk;
    return up(span, T) + (span + p.sinks <= Sk ? up(p.sinks, T) : 0);
  };
  p.wide = U <= kTokenGrid;
  if (p.token) {
    // A step of a workgroup's waves takes 1.1 us, joining parts 4: parts of five steps or more, for more than ten.
    const int64_t waves = (dh == 128 ? 2 : 4) * (p.wide ? 2 : 1), steps = up(tiles(R, TOKEN_KEYS), waves);
    p.fwd_parts = steps > 10 ? parts_for(U, steps, kTokenGrid, 5) : 1;
  } else p.fwd_parts = parts_for(U * up(R, OWN * 4), tiles(OWN * 4, TILE), 512, 4);
  p.q_parts = parts_for(U * up(R, OWN * 4), tiles(OWN * 4, TILE), 512, 4);
  const int64_t seen = (p.window + OWN * 4) * share < R ? (p.window + OWN * 4) * share : R;
  p.kv_parts = parts_for(U * up(Sk, OWN * 4), up(seen, TILE), 256, 4);
  // sinks that windows leave: 512 workgroups, each with 8 rounds of its waves' 32 rows or more
  p.sink_blocks = p.sinks && p.window < Sk ? (int)up(p.sinks, OWN) : 0;
  p.sink_parts = p.sink_blocks ? parts_for(U * p.sink_blocks, up(R, 4 * OWN), 512, 8) : 0;
  // threads of the largest launch, a sequence; of blocks that are dealt out in groups (deal) up to eight for seven more
  auto dealt = [&](int64_t blocks, int parts) { const int64_t n = blocks * parts; return Hkv * (n + (n < 8 ? n : 8) - 1); };
  auto larger = [](int64_t x, int64_t y) { return x > y ? x : y; };
  int64_t threads;
  if (backward) {
    threads = 256 * (dealt(up(Sk, OWN * 4), p.kv_parts) + dealt(up(R, OWN * 4), p.q_parts) + Hkv * p.sink_blocks * p.sink_parts);
    threads = larger(threads, Hkv * p.Rp * (dh / 8));
    if (p.kv_parts > 1) threads = larger(threads, Hkv * Sk * (dh / 4));
  } else {
    threads = p.token ? 512 * dealt(1, p.fwd_parts) : 256 * dealt(up(R, OWN * 4), p.fwd_parts);
    if (p.fwd_parts > 1) threads = larger(threads, Hkv * R * dh);
  }
  if (threads > kMostThreads) return false;
  p.at_once = (int)(B < kMostThreads / threads ? B : kMostThreads / threads);
  auto round = [](size_t b) { return (b + 255) / 256 * 256; };
  const bool parts = p.fwd_parts > 1;
  const size_t units = (size_t)p.at_once * Hkv;             // the next launch's sequences have the memory of those before
  p.fwd_ml = parts ? round(4 * p.fwd_parts * units * R * dh) : 0;
  p.fwd_bytes = parts ? p.fwd_ml + round(8 * p.fwd_parts * units * R) : 0;
  p.d = round(4 * units * p.Rp);
  p.part = 2 * p.d;
  p.kv_part = p.part + (p.q_parts > 1 ? round(4 * p.q_parts * units * R * dh) : 0);
  p.sink_part = p.kv_part + (p.kv_parts > 1 ? round(8 * p.kv_parts * units * Sk * dh) : 0);
  p.bwd_bytes = p.sink_part + (p.sink_parts > 1 ? round(8 * p.sink_parts * units * p.sinks * dh) : 0);
  return true;
}

WinArgs common_args(const WinPlan& p, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* start,
                    const int32_t* length, int B, int Sq, int Sk, int H, int Hkv, int dh) {
  WinArgs a{};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.start = start; a.length = length;
  a.B = B; a.Sq = Sq; a.Sk = Sk; a.share = H / Hkv; a.Hkv = Hkv; a.R = p.R; a.Rp = p.Rp;
  a.window = p.window; a.sinks = p.sinks; a.ring = Sk - p.sinks;
  a.scale = 1.0f / sqrtf((float)dh);
  a.c2 = 1.4426950408889634f * a.scale;
  return a;
}

// the sequences from b0 on, as many as go into a launch; the work memory of those before is free when they are done
WinArgs sequences(WinArgs a, const WinPlan& p, int b0) {
  const int64_t q = (int64_t)b0 * a.Sq, k = (int64_t)b0 * a.Sk;
  a.B = a.B - b0 < p.at_once ? a.B - b0 : p.at_once;
  a.q += q * a.ldq; a.k += k * a.ldk; a.v += k * a.ldv;
  if (a.start) a.start += b0;
  if (a.length) a.length += b0;
  a.lse2 += (int64_t)b0 * a.Hkv * a.R;
  if (a.out) a.out += q * a.ldo;
  if (a.o) { a.o += q * a.ldo; a.dout += q * a.lddo; a.dq += q * a.lddq; a.dk += k * a.lddk; a.dv += k * a.lddv; }
  return a;
}

template <int DH, bool WIDE>
rv_status tokens(WinArgs& a, const WinPlan& p, hipStream_t st) {
  constexpr int waves = kTokenWaves<DH, WIDE>, ring = waves * kTokenRing<DH>, image = waves * (DH / 2 * 64 * 4 + 32 * 8);
  const int64_t grid = deal(a.fwd, a, a.start || a.length, 1, p.fwd_parts);
  return launch<window_token_kernel<DH, waves>>(a, grid, 64 * waves, ring > image ? ring : image, st);
}
template <int DH>
rv_status forward(WinArgs a, const WinPlan& p, char* work, hipStream_t st) {
  const int64_t U = (int64_t)a.B * a.Hkv;
  const bool unequal = a.start || a.length;
  a.part = (float*)work; a.part_ml = (float2*)(work + p.fwd_ml);
  if (p.token) {
    RV_TRY((p.wide ? tokens<DH, true>(a, p, st) : tokens<DH, false>(a, p, st)));
  } else {
    const int64_t grid = deal(a.fwd, a, unequal, up(a.R, OWN * 4), p.fwd_parts);
    // Narrow windows 32 keys at a time: what a wave's own tokens do not see is left out, and heads of 64 take 117 registers, four waves to a SIMD.  us, 32 / 64
    // keys: 4 x 2000 tokens of 16 heads of 64, windows of 64 / 256 / 512 / 1024 / 1500: 18 / 21, 25 / 32, 35 / 42, 53 / 55, 70 / 63; of 128 34 / 34, 45 / 44,
    // 58 / 57, 85 / 82, 105 / 98; 4 x 4000 of 16 heads over 2 of 128, windows of 64 / 256 / 512 / 1024: 47 / 50, 77 / 80, 104 / 103, 154 / 148.  Heads of 128 gain 6 %
    // at a window of 64 and lose 4 at 1024; between 256 and 512 the two are within 4 % of each other either way, and the border could be anywhere there.  (Tiles
    // of 32 in rings of 3 and 4 in place of 64 in two: 3 to 10 % slower, by their barriers.)
    if (a.window <= (DH == 64 ? 1024 : 512)) RV_TRY((launch<window_fwd_kernel<DH, 4, 2, 1>>(a, grid, 256, 2 * 2 * kTileBytes<DH>, st)));
    else RV_TRY((launch<window_fwd_kernel<DH, 4, 2, 2>>(a, grid, 256, 2 * 2 * kTileBytes<DH>, st)));
  }
  if (p.fwd_parts == 1) return RV_OK;
  if (p.fwd_parts > 4) RV_TRY((launch<window_join_kernel<DH, 8>>(a, up(U * a.R * (DH / 8), 32), 256, 0, st)));
  else RV_TRY((launch<window_join_kernel<DH, 1>>(a, up(U * a.R * (DH / 8), 256), 256, 0, st)));
  return RV_OK;
}
template <int DH, int NW, int NS, int ROWS, int NS_Q>
rv_status backward(WinArgs a, const WinPlan& p, char* work, hipStream_t st) {
  const int64_t U = (int64_t)a.B * a.Hkv;
  a.stat_lse = (float*)work; a.stat_d = (float*)(work + p.d); a.q_part = (float*)(work + p.part); a.kv_part = (float*)(work + p.kv_part);
  a.sink_part = (float*)(work + p.sink_part); a.sink_blocks = p.sink_blocks; a.sink_parts = p.sink_parts;
  RV_TRY((launch<window_stat_kernel<DH>>(a, up(U * a.Rp * (DH / 8), 256), 256, 0, st)));
  const int64_t kv = deal(a.bkv, a, a.length != nullptr, up(a.Sk, OWN * NW), p.kv_parts);
  const int64_t q = deal(a.bq, a, a.length != nullptr, up(a.R, OWN * NW), p.q_parts);
  a.kv_grid = (int)kv; a.sink_grid = (int)(U * p.sink_blocks * p.sink_parts);
  RV_TRY((launch<window_bwd_kernel<DH, NW, NS, ROWS, NS_Q>>(a, kv + a.sink_grid + q, 64 * NW, kBwdLds<DH, NW, NS, ROWS, NS_Q>, st)));
  if (p.q_parts > 1) RV_TRY((launch<window_bwd_join_kernel<DH, false>>(a, up(U * a.R * (DH / 8), 256), 256, 0, st)));
  if (p.kv_parts > 1 || p.sink_parts > 1) RV_TRY((launch<window_bwd_join_kernel<DH, true>>(a, up(U * (p.kv_parts > 1 ? a.Sk : a.sinks) * (DH / 4), 256), 256, 0, st)));
  return RV_OK;
}

}  // namespace

extern "C" rv_status rv_k_window_attention_work(int B, int Sq, int Sk, int n_heads, int n_kv_heads, int d_head, int window, int sinks, int backward,
                                                size_t* bytes) {
  WinPlan p;
  if (!bytes || !make_plan(p, B, Sq, Sk, n_heads, n_kv_heads, d_head, window, sinks, backward != 0)) return RV_E_INVAL;
  *bytes = backward ? p.bwd_bytes : p.fwd_bytes;
  return RV_OK;
}

extern "C" rv_status rv_k_window_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* start,
                                               const int32_t* length, void* out, int64_t ldo, float* lse2, int B, int Sq, int Sk, int n_heads,
                                               int n_kv_heads, int d_head, int window, int sinks, void* work, size_t work_bytes, void* stream) {
  WinPlan p;
  if (!make_plan(p, B, Sq, Sk, n_heads, n_kv_heads, d_head, window, sinks, false) || (!start && Sk < Sq)) return RV_E_INVAL;
  const int64_t cols = (int64_t)n_heads * d_head, kcols = (int64_t)n_kv_heads * d_head;
  if (bad(q, 16) || bad(k, 16) || bad(v, 16) || bad(out, 16) || bad(lse2, 4) || (((uintptr_t)start | (uintptr_t)length) & 3)) return RV_E_INVAL;
  if (bad_pitch(ldq, cols) || bad_pitch(ldk, kcols) || bad_pitch(ldv, kcols) || bad_pitch(ldo, cols)) return RV_E_INVAL;
  if (p.fwd_bytes && (bad(work, 256) || work_bytes < p.fwd_bytes)) return RV_E_INVAL;
  WinArgs a = common_args(p, q, ldq, k, ldk, v, ldv, start, length, B, Sq, Sk, n_heads, n_kv_heads, d_head);
  a.out = (uint16_t*)out; a.ldo = ldo; a.lse2 = lse2;
  for (int b = 0; b < B; b += p.at_once) {
    const WinArgs some = sequences(a, p, b);
    RV_TRY(d_head == 64 ? forward<64>(some, p, (char*)work, (hipStream_t)stream) : forward<128>(some, p, (char*)work, (hipStream_t)stream));
  }
  return RV_OK;
}

extern "C" rv_status rv_k_window_attention_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* length,
                                               const void* out, int64_t ldo, const void* dout, int64_t lddo, const float* lse2, void* dq, int64_t lddq,
                                               void* dk, int64_t lddk, void* dv, int64_t lddv, int B, int S, int n_heads, int n_kv_heads, int d_head,
                                               int window, int sinks, void* work, size_t work_bytes, void* stream) {
  WinPlan p;
  if (!make_plan(p, B, S, S, n_heads, n_kv_heads, d_head, window, sinks, true)) return RV_E_INVAL;
  const int64_t cols = (int64_t)n_heads * d_head, kcols = (int64_t)n_kv_heads * d_head;
  if (bad(q, 16) || bad(k, 16) || bad(v, 16) || bad(out, 16) || bad(dout, 16) || bad(lse2, 4) || bad(dq, 16) || bad(dk, 16) || bad(dv, 16) ||
      ((uintptr_t)length & 3)) return RV_E_INVAL;
  if (bad_pitch(ldq, cols) || bad_pitch(ldk, kcols) || bad_pitch(ldv, kcols) || bad_pitch(ldo, cols) || bad_pitch(lddo, cols) || bad_pitch(lddq, cols) ||
      bad_pitch(lddk, kcols) || bad_pitch(lddv, kcols)) return RV_E_INVAL;
  if (bad(work, 256) || work_bytes < p.bwd_bytes) return RV_E_INVAL;
  WinArgs a = common_args(p, q, ldq, k, ldk, v, ldv, nullptr, length, B, S, S, n_heads, n_kv_heads, d_head);
  a.o = (const uint16_t*)out; a.ldo = ldo; a.dout = (const uint16_t*)dout; a.lddo = lddo; a.lse2 = (float*)lse2;
  a.dq = (uint16_t*)dq; a.lddq = lddq; a.dk = (uint16_t*)dk; a.lddk = lddk; a.dv = (uint16_t*)dv; a.lddv = lddv;
  for (int b = 0; b < B; b += p.at_once) {
    const WinArgs some = sequences(a, p, b);
    RV_TRY(d_head == 64 ? (backward<64, 4, 2, 64, 2>(some, p, (char*)work, (hipStream_t)stream))
                        : (backward<128, 4, 2, 32, 2>(some, p, (char*)work, (hipStream_t)stream)));
  }
  return RV_OK;
}

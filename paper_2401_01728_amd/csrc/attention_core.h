// What attention kernels share whose streamed side goes global -> LDS in tiles of 64 rows of heads of 64 or 128 columns: tiles without bank
// conflicts for reads of whole rows and for transposing reads, fragments, and the loads and stores of a wave's own rows.
#pragma once
#include "gemm_core.h"

namespace {

constexpr int TILE = 64;                 // streamed rows
constexpr int OWN = 32;                  // rows or keys a wave owns

typedef __bf16 Frag __attribute__((ext_vector_type(8)));

// row of a tile -> what its chunk indexes are xor-ed with.  Rows of 128 columns (16 chunks, one bank line of 256 bytes): a permutation of 16
// over 16 rows, for the reads of one chunk of 16 rows, whose upper two bits differ among four neighbouring rows, for the transposing reads of 64
// bytes of four rows.  64 columns: two rows to a line, so eight values over 16 rows and one bit among the rows of a parity.
template <int DH>
__device__ __forceinline__ int swizzle(int row) {
  return DH == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}
template <int DH> constexpr int kTileBytes = TILE * DH * 2;

// A fragment, rows row0 + lane % 32, columns 16 kk + 8 (lane / 32) .. + 7
template <int DH>
__device__ __forceinline__ Frag frag_rows(const char* lds, int row0, int kk) {
  const int l = threadIdx.x & 63, row = row0 + (l & 31);
  return *reinterpret_cast<const Frag*>(lds + row * (DH * 2) + (((kk * 2 + (l >> 5)) ^ swizzle<DH>(row)) << 4));
}
// A fragment of the transposed tile: m = column col0 + lane % 32, its eight k the rows row0 + 4 g + (0 .. 3) and row0 + 8 + 4 g + (0 .. 3) of
// lane group g = lane / 32 - those of a lane's accumulator registers
template <int DH>
__device__ __forceinline__ Frag frag_cols(const char* lds, int row0, int col0) {
  const int l = threadIdx.x & 63, q = l >> 4, i = l & 15;
  const int row = row0 + 4 * (q >> 1) + (i >> 2), col = col0 + 16 * (q & 1) + 4 * (i & 3);
  auto at = [&](int r) {
    return (s16x4 __attribute__((address_space(3)))*)(lds + r * (DH * 2) + (((col >> 3) ^ swizzle<DH>(r)) << 4) + (col & 7) * 2);
  };
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(row)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(row + 8));
  return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// N products in a row whose A fragments come from LDS: fragment i is asked for DEPTH products before its own.  (Left to itself the compiler reads
// each one right in front of its product and waits out the latency of LDS every time.)
template <int N, int DEPTH, typename Load, typename Use>
__device__ __forceinline__ void in_a_row(Load load, Use use) {
  decltype(load(0)) f[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH && i < N; ++i) f[i] = load(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    use(i, f[i % DEPTH]);
    if (i + DEPTH < N) f[i % DEPTH] = load(i + DEPTH);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// what was loaded from memory is there behind this point: a wait for it inside a loop would wait for the loads of tiles, too
template <int N>
__device__ __forceinline__ void settle(Frag (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}
// registers 8 ks .. 8 ks + 7 of an accumulator, rounded: a B fragment
__device__ __forceinline__ Frag pack_frag(const f32x16& a, int ks) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = rv_pack_bf16x2(a[8 * ks + 2 * i], a[8 * ks + 2 * i + 1]);
  return __builtin_bit_cast(Frag, r);
}
// streamed row (of 32) of accumulator register r in lane group g
__device__ __forceinline__ int acc_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

template <int N>
__device__ __forceinline__ void clear(f32x16 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) v[i][r] = 0.f;
}

// waits that later LDS reads are not moved in front of
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// A wave's share of the loads of a tile of ROWS rows: load i of lane l is chunk (i NW + wave) 64 + l of the tile in LDS.  A load brings STEP rows
// further than the one before; where that is a multiple of the swizzle's period all of a lane's loads have one column.
template <int DH, int NW, int ROWS = TILE>
struct TileLoads {
  static constexpr int N = ROWS * DH / 8 / 64 / NW, STEP = NW * 64 / (DH / 8);
  static constexpr bool kOneColumn = STEP % 16 == 0;
  int row, col[kOneColumn ? 1 : N];                      // first row; columns in elements
  int wave;
  __device__ __forceinline__ explicit TileLoads(int w) : wave(w) {
    const int slot = wave * 64 + (threadIdx.x & 63);
    row = slot / (DH / 8);
#pragma unroll
    for (int i = 0; i < (kOneColumn ? 1 : N); ++i) col[i] = ((slot % (DH / 8)) ^ swizzle<DH>(row + i * STEP)) * 8;
  }
  __device__ __forceinline__ int column(int i) const { return col[kOneColumn ? 0 : i]; }
  // keys k0 .. of a sequence of n, clamped to the last one
  __device__ __forceinline__ void keys(const uint16_t* base, int64_t ld, int k0, int n, char* lds) const {
    const int m0v = __builtin_amdgcn_readfirstlane((int)(size_t)lds + wave * 1024);
    const uint16_t* from = base + (int64_t)k0 * ld;
    const int last = n - 1 - k0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row + i * STEP < last ? row + i * STEP : last;
      dtl_load_s(from, (unsigned)r * (unsigned)(ld * 2) + column(i) * 2, m0v + i * NW * 1024);
    }
  }
  // rows r0 .. of the list of a key/value head's query rows, clamped to the last of R, of two matrices; place(r): the token, and the column in
  // front of column(i), of row r
  template <typename Place>
  __device__ __forceinline__ void rows(Place place, int R, const uint16_t* q, int64_t ldq, const uint16_t* o, int64_t ldo, int r0, char* lds_q, char* lds_o) const {
    const int mq = __builtin_amdgcn_readfirstlane((int)(size_t)lds_q + wave * 1024), mo = __builtin_amdgcn_readfirstlane((int)(size_t)lds_o + wave * 1024);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r = r0 + row + i * STEP;
      r = r < R ? r : R - 1;
      int64_t tok;
      int c;
      place(r, tok, c);
      c += column(i);
      const uint16_t* pq = q + tok * ldq + c;
      const uint16_t* po = o + tok * ldo + c;
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(pq), "s"(mq + i * NW * 1024) : "memory", "m0");
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(po), "s"(mo + i * NW * 1024) : "memory", "m0");
    }
  }
};
// 64 floats -> LDS
__device__ __forceinline__ void load_floats(const float* from, char* lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               : : "v"((threadIdx.x & 63) * 4), "s"(from), "s"(__builtin_amdgcn_readfirstlane((int)(size_t)lds)) : "memory", "m0");
}

// a wave's owned rows as B fragments
template <int DH>
__device__ __forceinline__ void load_owned(Frag (&f)[DH / 16], const uint16_t* row) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) f[kk] = *reinterpret_cast<const Frag*>(row + kk * 16 + (l >> 5) * 8);
}
// acc^T (lane = row) as bf16, or as it is
template <int DH>
__device__ __forceinline__ void store_owned(const f32x16 (&acc)[DH / 32], float mul, uint16_t* row) {
  const int grp = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) {
      u32x2 o;
      o.x = rv_pack_bf16x2(acc[dt][4 * rg] * mul, acc[dt][4 * rg + 1] * mul);
      o.y = rv_pack_bf16x2(acc[dt][4 * rg + 2] * mul, acc[dt][4 * rg + 3] * mul);
      *reinterpret_cast<u32x2*>(row + dt * 32 + 8 * rg + 4 * grp) = o;
    }
}
template <int DH>
__device__ __forceinline__ void store_owned32(const f32x16 (&acc)[DH / 32], float* row) {
  const int grp = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *reinterpret_cast<f32x4*>(row + dt * 32 + 8 * rg + 4 * grp) =
          f32x4{acc[dt][4 * rg], acc[dt][4 * rg + 1], acc[dt][4 * rg + 2], acc[dt][4 * rg + 3]};
}

// A row of one key: its probability is 1 whatever the score, so the score's gradient is zero; what stands here is the difference of one sum
// formed in two orders.  (Times zero: what is not a number stays none.)
template <int N>
__device__ __forceinline__ void of_one_key(f32x16 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] *= 0.f;
}

// blocks of rows or keys of a (sequence, key/value head), parts of the streamed side, and how the list of them is dealt out (where)
struct Grid { int blocks, parts, groups; };

// Workgroup -> (sequence, key/value head, part, block): ids go to the 8 XCDs in turn; each takes a contiguous range of a list in which the
// blocks of one (head, sequence), which read the same keys, are neighbours.  Where sequences have lengths of their own a range has to hold as
// much of each as any other: the list then goes through the heads, or through `groups` equal shares of a head's blocks where
// there are fewer than eight heads or no multiple of it, and has a share's blocks of every sequence behind one another (16 heads over 4, lengths of
// 2048 .. 0: 238 us with whole heads, 232 with halves).
__host__ __device__ inline int share_of(const Grid& g) { return (g.blocks * g.parts + g.groups - 1) / g.groups; }
struct Where { int b, h, part, block, unit; };
template <typename Args>
__device__ __forceinline__ bool where(const Args& a, const Grid& g, int id, int total, Where& w) {
  const int base = total / 8, rem = total % 8, x = id % 8, share = share_of(g);
  const int v = x * base + (x < rem ? x : rem) + id / 8;
  int u = v / share;
  w.b = u % a.B; u /= a.B;
  w.h = u / g.groups;
  const int i = u % g.groups * share + v % share;
  w.part = i / g.blocks;
  w.block = i - w.part * g.blocks;
  w.unit = w.b * a.Hkv + w.h;
  return w.part < g.parts;
}

// ---- host ----
inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kMostParts = 64;

// Parts of the streamed side: as many as give `want` workgroups, each with `least` tiles or more.
int parts_for(int64_t blocks, int64_t tiles, int64_t want, int64_t least) {
  int64_t p = want / (blocks > 0 ? blocks : 1);
  if (p > tiles / least) p = tiles / least;
  return (int)(p < 1 ? 1 : p > kMostParts ? kMostParts : p);
}

// A launch of the runtime has fewer than 2^32 threads; a call of more is made for some of its sequences at a time.
constexpr int64_t kMostThreads = 3ll << 30;

template <auto Kern, typename Args>
rv_status launch(const Args& a, int64_t grid, int threads, int lds, hipStream_t st) {
  if (rv_allow_lds<Kern>(lds) != hipSuccess) return RV_E_DEVICE;
  hipLaunchKernelGGL(Kern, dim3((unsigned)grid), dim3(threads), lds, st, a);
  return rv_launch_status();
}

bool bad(const void* p, uintptr_t to) { return !p || ((uintptr_t)p & (to - 1)); }
bool bad_pitch(int64_t ld, int64_t cols) { return ld < cols || ld % 8 || ld > (1 << 24); }

// the launch of `blocks` x parts per (sequence, key/value head); unequal: sequences may have lengths of their own
template <typename Args>
int64_t deal(Grid& g, const Args& a, bool unequal, int64_t blocks, int parts) {
  g.blocks = (int)blocks; g.parts = parts; g.groups = 1;
  if (unequal && a.B > 1) {
    while (g.groups < 8 && a.Hkv * g.groups % 8) g.groups *= 2;
    if (g.groups > blocks * parts) g.groups = (int)(blocks * parts);
  }
  return (int64_t)a.B * a.Hkv * g.groups * share_of(g);
}

}  // namespace

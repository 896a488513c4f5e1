// Shared parts of the attention kernels (attn.hip, attn_back.hip): the batch's
// rows, operand tiles in LDS and the 32 x 32 bf16 MFMA.
#pragma once

#include "common.h"

namespace dr {
namespace attn {

constexpr int kThreads = 256;          // four waves
constexpr int kWaves = 4;
constexpr int kRows = 128;             // rows of a workgroup's own tile: 32 a wave
constexpr int kFewRows = 32;           // where there are few tiles

// 32x32x16 bf16 MFMA, fp32 accumulate.  Lane l supplies A[l % 32][8 (l / 32) ..
// + 8] and B[8 (l / 32) .. + 8][l % 32]; register r of lane l holds
// C[8 (r / 4) + 4 (l / 32) + r % 4][l % 32].
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Two values as bf16, rounded to nearest even, a in the low half.  (Written for
// the compiler and not as asm: a result of exp2 needs a wait state before the
// next instruction reads it, which the compiler does not add in front of asm.)
__device__ __forceinline__ unsigned pack2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// row of C that register r holds, less 4 (l / 32)
__device__ __forceinline__ constexpr int c_row(int r) { return 8 * (r >> 2) + (r & 3); }
// On a 32 x 32 tile whose rows and columns are the same tokens: `v` where the row
// comes after the lane's column (AFTER), or before it.  The lanes are a constant of
// the register, so a value costs one selection and no comparison.
constexpr unsigned long long diagonal_lanes(int r, bool after) {
  unsigned long long m = 0;
  for (int l = 0; l < 64; ++l) {
    const int row = c_row(r) + 4 * (l >> 5), col = l & 31;
    if (after ? row > col : row < col) m |= 1ull << l;
  }
  return m;
}
template <bool AFTER, int R = 0>
__device__ __forceinline__ void mask_diagonal(f32x16& c, float v) {
  constexpr unsigned long long lanes = diagonal_lanes(R, AFTER);
  c[R] = __builtin_amdgcn_inverse_ballot_w64(lanes) ? v : c[R];
  if constexpr (R < 15) mask_diagonal<AFTER, R + 1>(c, v);
}
// Registers 8 s .. 8 s + 7 of a C tile as the B operand of step s (16 of the
// tile's 32 rows): half h of the wave holds rows 16 s + {4 h .. + 3, 8 + 4 h ..
// + 3}, and the A operand takes its eight columns in the same order (two
// transposing LDS reads, read_cols), so no value changes lanes.
__device__ __forceinline__ u32x4 c_operand(const f32x16& c, int s) {
  return u32x4{pack2(c[8 * s], c[8 * s + 1]), pack2(c[8 * s + 2], c[8 * s + 3]),
               pack2(c[8 * s + 4], c[8 * s + 5]), pack2(c[8 * s + 6], c[8 * s + 7])};
}

// LDS tile of rows of D bf16: segment (16 bytes) seg of row r in slot
// seg ^ tile_swz(r).  Read either by rows (read_rows: 32 rows, one segment per
// half wave) or transposed (read_cols: four rows by 16 columns per group of
// 16 lanes); both take every bank equally often: 16 rows put one segment into 16
// different slots of the 256 bytes that the banks hold, and rows 4 m .. 4 m + 3
// put four segments into different 64-byte quarters.
template <int D>
__device__ __forceinline__ int tile_swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
// A lane's place in a tile for both kinds of reads.  The step (32 bytes of a
// row), the column block (64 bytes) and the second group of four rows each are
// one exclusive-or with it, rows further down an immediate offset: begin() makes
// the two registers of a stage opaque, since the compiler otherwise keeps every
// such address in a register of its own over the whole loop, and spills them.
template <int D>
struct TilePlace {
  unsigned rows, cols;   // bytes from the tile's start
  __device__ __forceinline__ void init(int lane) {
    const int r = lane & 31, h = lane >> 5, q = (lane >> 2) & 3, s0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    rows = (unsigned)(r * 2 * D + ((h ^ tile_swz<D>(r)) << 4));
    cols = (unsigned)((4 * h + q) * 2 * D + ((D == 128 ? q : q >> 1) << 6) + ((s0 ^ h) << 4) + (lane & 1) * 8);
  }
  __device__ __forceinline__ TilePlace begin(unsigned stage) const {
    TilePlace p = {rows + stage, cols + stage};
    asm volatile("" : "+v"(p.rows), "+v"(p.cols));
    return p;
  }
};
// A operand [32 rows from row0][16 columns of step ks] of the tile at `tile`
template <int D>
__device__ __forceinline__ u32x4 read_rows(const unsigned char* lds, const TilePlace<D>& p, int tile, int row0, int ks) {
  return *reinterpret_cast<const u32x4*>(lds + (p.rows ^ (ks << 5)) + (tile + row0 * 2 * D));
}
// A operand [32 columns of block cb][16 rows from row0, in c_operand's order]
template <int D>
__device__ __forceinline__ u32x4 read_cols(const unsigned char* lds, const TilePlace<D>& p, int tile, int row0, int cb) {
  const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr16(lds + (p.cols ^ (cb << 6)) + (tile + row0 * 2 * D)));
  const uint2 hi = __builtin_bit_cast(uint2, lds_read_tr16(lds + (p.cols ^ 32 ^ (cb << 6)) + (tile + (row0 + 8) * 2 * D)));
  return u32x4{lo.x, lo.y, hi.x, hi.y};
}

// Fills a tile of R rows from rows of `ldb` bytes by LDS DMA: each instruction of
// a wave moves 1 KB (64 / (D / 8) rows).  Rows past `rows` (which may be negative)
// read as zeros: the descriptor ends after the last row.
template <int D, int R, int WAVES = kWaves>
struct TileLoad {
  static constexpr int kPer = 512 / D;              // rows per instruction
  static constexpr int kCount = R / kPer / WAVES;   // instructions per wave
  static_assert(kCount >= 1, "a wave moves at least 1 KB");
  unsigned voff[kCount];
  __device__ __forceinline__ void init(int w, int lane, unsigned ldb) {
#pragma unroll
    for (int u = 0; u < kCount; ++u) {
      const int r = (w + WAVES * u) * kPer + lane / (D / 8);
      voff[u] = (unsigned)r * ldb + (unsigned)(((lane % (D / 8)) ^ tile_swz<D>(r)) << 4);
    }
  }
  __device__ __forceinline__ void issue(const unsigned char* base, int rows, unsigned ldb, unsigned dst, int w) const {
    const int n = rows < R ? rows : R;
    const unsigned bytes = n > 0 ? (unsigned)(n - 1) * ldb + 2 * D : 0u;
    const unsigned long long b = reinterpret_cast<unsigned long long>(base);
    const u32x4 rsrc = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)b),
                        (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(b >> 32)) & 0xffffu,
                        (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
#pragma unroll
    for (int u = 0; u < kCount; ++u)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :: "s"(dst + (w + WAVES * u) * 1024), "v"(voff[u]), "s"(rsrc) : "memory", "m0");
  }
};

// Loaded values are in their registers from here on.  Without it the compiler
// waits for them at their first use, inside the loop, on every turn; and since
// loads end in order, that wait would cover the DMA that the turn has just issued.
__device__ __forceinline__ void arrived(u32x4& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void arrived(float& v) { asm volatile("" : "+v"(v)); }

// B operand fragments of one row per lane (row l % 32 of the wave's 32): the
// D / 16 steps' eight columns from 16 s + 8 (l / 32); zeros where !ok
template <int D>
__device__ __forceinline__ void row_fragments(const unsigned char* row, bool ok, int lane, u32x4 (&f)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) f[s] = u32x4{0u, 0u, 0u, 0u};
  if (ok) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      f[s] = *reinterpret_cast<const u32x4*>(row + 32 * s + 16 * (lane >> 5));
  }
}

// The same out of the wave's own 32 rows in LDS (TileLoad by one wave)
template <int D>
__device__ __forceinline__ void tile_fragments(const unsigned char* tile, const TilePlace<D>& p, u32x4 (&f)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) f[s] = read_rows<D>(tile, p, 0, 0, s);
}

// The batch: sequence i holds rows [first, first + len) of the tensors and its
// slot ends at `end` (first of the next one; the last slot ends with the rows).
struct Batch {
  const int* off;     // [N + 1], or NULL: sequence i starts at row i T
  const int* len;     // [N], or NULL: the whole slot
  long long rows, T;
  int N;
};
struct Seq {
  long long first, end;
  int len;
};
// A packed slot's ends, clamped into the rows: the slots of ascending offsets then take
// every row at most once, whatever their values (what the grid of listed places rests on).
__device__ __forceinline__ void clamp_slot(const Batch& b, long long& first, long long& next) {
  first = first < 0 ? 0 : (first > b.rows ? b.rows : first);
  next = next < first ? first : (next > b.rows ? b.rows : next);
}
// Values outside their range are clamped: no row outside [0, rows) is touched.  (i
// is uniform; the constant address space makes these scalar loads, which do not
// queue behind the vector loads of the waves around.)
__device__ __forceinline__ Seq sequence(const Batch& b, int i) {
  typedef const __attribute__((address_space(4))) int* Ints;
  const int u = __builtin_amdgcn_readfirstlane(i);
  Seq s;
  long long next;
  const int given = b.len ? ((Ints)b.len)[u] : 0x7fffffff;
  if (b.off) {
    s.first = ((Ints)b.off)[u];
    next = ((Ints)b.off)[u + 1];
    clamp_slot(b, s.first, next);
  } else {
    s.first = i * b.T;
    next = s.first + b.T;
  }
  s.end = i == b.N - 1 ? b.rows : next;
  long long n = next - s.first;
  if (n > b.T) n = b.T;
  if (given < n) n = given < 0 ? 0 : given;
  s.len = (int)n;
  return s;
}

// A launch's work: pairs of a sequence and a place (tile index) in it, for each key
// head and `per` workgroups on it.  Workgroup x of a row of the grid runs on XCD
// x % 8.  An XCD takes the key heads of its own class (E classes, the largest of 8,
// 4, 2, 1 that divides Hkv), so that keys and values are read through one L2, or
// 8 / E of them; the 8 / E XCDs of a class take the items in turn.  Places go from
// the highest, the longest work, down.  The items are all N * tiles pairs, most of
// which may be empty where a few packed sequences are much longer than the others;
// then (`listed`) every workgroup finds its own among those that the slots have.
// 61 sequences of 1 to 2039 tokens: 2640 workgroups instead of 15616, 1 us less per
// thousand.
// (Divisions by numbers of the launch are products: x / d = x m >> shift.)
struct Divisor {
  unsigned d, m, shift;
};
__device__ __forceinline__ unsigned over(unsigned x, const Divisor& v) {   // x < 2^31
  return (unsigned)(((unsigned long long)x * v.m) >> v.shift);
}
struct Grid {
  int items, tiles, class_bits, own, listed;   // class_bits: log2 E; own: rows of a tile
  Divisor N, per;
};
struct Place {
  int seq, place, khead, g, tiles;   // tiles: of this sequence's slot
};
constexpr int kListed = 256;         // most sequences that a wave looks through: four a lane

__device__ __forceinline__ int wave_total(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast31 into rows 2 and 3
  return __builtin_amdgcn_readlane(v, 63);
}
// The item-th pair of a sequence and a place that its slot has, by descending place.
__device__ __forceinline__ bool listed_place(const Grid& q, const Batch& b, int item, Place& p) {
  const int lane = threadIdx.x & 63;
  int nt[kListed / 64];   // tiles of this lane's sequences (lane, lane + 64, ..); the last slot has one at least
#pragma unroll
  for (int j = 0; j < kListed / 64; ++j) {
    const int i = lane + 64 * j;
    nt[j] = 0;
    if (i < b.N) {
      long long first = b.off[i], next = b.off[i + 1];
      clamp_slot(b, first, next);
      const long long n = next - first < b.T ? next - first : b.T;
      nt[j] = (int)((n + q.own - 1) / q.own);
      if (i == b.N - 1 && nt[j] == 0) nt[j] = 1;
    }
  }
  auto from = [&](int place) {   // pairs with this place or a higher one
    int n = 0;
#pragma unroll
    for (int j = 0; j < kListed / 64; ++j) n += nt[j] > place ? nt[j] - place : 0;
    return wave_total(n);
  };
  int lo = 0, hi = q.tiles, above = 0;   // from(lo) > item >= from(hi) = above
  if (from(0) <= item) return false;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, n = from(mid);
    if (n > item) lo = mid;
    else hi = mid, above = n;
  }
  int rank = item - above;
  p.place = lo;
  p.seq = 0;
  p.tiles = 1;
#pragma unroll
  for (int j = 0; j < kListed / 64; ++j) {
    const unsigned long long has = __ballot(nt[j] > lo);
    const int n = __popcll(has);
    if (rank >= 0 && rank < n) {
      const int before = __popcll(has & ((1ull << lane) - 1));
      const int at = __ffsll((unsigned long long)__ballot(nt[j] > lo && before == rank)) - 1;
      p.seq = 64 * j + at;
      p.tiles = __builtin_amdgcn_readlane(nt[j], at);
    }
    rank -= n;
  }
  return true;
}
__device__ __forceinline__ bool place_of(const Grid& q, const Batch& b, Place& p) {
  const int x = blockIdx.x & 7, s = blockIdx.x >> 3;
  const long long item = (((long long)blockIdx.z * gridDim.y + blockIdx.y) << (3 - q.class_bits)) + (x >> q.class_bits);
  if (item >= q.items) return false;
  const int h = (int)over((unsigned)s, q.per);
  p.g = s - h * (int)q.per.d;
  p.khead = (h << q.class_bits) + (x & ((1 << q.class_bits) - 1));
  if (q.listed) return listed_place(q, b, (int)item, p);
  const int down = (int)over((unsigned)item, q.N);
  p.seq = (int)item - down * (int)q.N.d;
  p.place = q.tiles - 1 - down;
  p.tiles = q.tiles;
  return true;
}

// Zeros the rows [from, to) of a head: W bytes a row, by the whole workgroup
template <int W>
__device__ __forceinline__ void zero_rows(unsigned char* base, long long ldb, long long from, long long to) {
  constexpr int kPerRow = W / 16;
  for (long long i = from * kPerRow + threadIdx.x; i < to * kPerRow; i += blockDim.x)
    *reinterpret_cast<u32x4*>(base + i / kPerRow * ldb + i % kPerRow * 16) = u32x4{0u, 0u, 0u, 0u};
}

// C^T of a wave's 32 rows (row l % 32 per lane, column 32 cb + c_row(r) + 4 h in
// register r) as bf16, scaled: through the wave's own LDS (store_bytes of it), so
// that every store instruction writes whole rows.  (As the lanes hold it, each
// would write 32 pieces of 16 bytes, D / 8 pieces to a cache line.)
template <int D>
constexpr int store_bytes = 32 * (2 * D + 16);
template <int D>
__device__ __forceinline__ void store_rows(unsigned char* lds, unsigned char* rows, long long ldb, int n,
                                           const f32x16 (&acc)[D / 32], float scale, int lane) {
  unsigned char* mine = lds + (lane & 31) * (2 * D + 16) + 8 * (lane >> 5);
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint2*>(mine + 64 * cb + 16 * q) =
          uint2{pack2(acc[cb][4 * q] * scale, acc[cb][4 * q + 1] * scale),
                pack2(acc[cb][4 * q + 2] * scale, acc[cb][4 * q + 3] * scale)};
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (a wave's own values: no barrier)
  constexpr int kPer = 512 / D;   // rows per store
  const int r0 = lane / (D / 8), seg = lane % (D / 8);
#pragma unroll
  for (int i = 0; i < 32 / kPer; ++i) {
    const int r = i * kPer + r0;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + r * (2 * D + 16) + 16 * seg);
    if (r < n) *reinterpret_cast<u32x4*>(rows + r * ldb + 16 * seg) = v;
  }
}

// The four waves' C^T of the same 32 rows, each scaled by its lane's f, summed in order
// and stored as bf16: through LDS (join_bytes), by the whole workgroup.
template <int D>
constexpr int join_bytes = kWaves * 32 * (4 * D + 16);
template <int D>
__device__ __forceinline__ void join_waves(unsigned char* lds, const f32x16 (&acc)[D / 32], float f, unsigned char* rows,
                                           long long ldb, int n, int w, int lane) {
  constexpr int kPitch = 4 * D + 16;
  unsigned char* mine = lds + (w * 32 + (lane & 31)) * kPitch + 16 * (lane >> 5);
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(mine + 128 * cb + 32 * q) =
          f32x4{acc[cb][4 * q] * f, acc[cb][4 * q + 1] * f, acc[cb][4 * q + 2] * f, acc[cb][4 * q + 3] * f};
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * (D / 8); i += kThreads) {
    const int r = i / (D / 8), seg = i % (D / 8);
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll
    for (int p = 0; p < kWaves; ++p) {
      const unsigned char* at = lds + (p * 32 + r) * kPitch + 32 * seg;
      x += *reinterpret_cast<const f32x4*>(at);
      y += *reinterpret_cast<const f32x4*>(at + 16);
    }
    if (r < n)
      *reinterpret_cast<u32x4*>(rows + r * ldb + 16 * seg) =
          u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3])};
  }
}

// v of lanes l and l ^ 32 joined, without LDS: two copies of v exchange halves
__device__ __forceinline__ float sum_halves(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ float max_halves(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// x / d for x < 2^31: with l = ceil(log2 d), m = floor(2^(31 + l) / d) + 1 < 2^32 is
// off by at most 1 / d of a quotient's unit
inline Divisor divisor(unsigned d) {
  unsigned l = 0;
  while ((1ull << l) < d) ++l;
  return Divisor{d, (unsigned)((1ull << (31 + l)) / d + 1), 31 + l};
}
// host side of Grid, for tiles of `own` rows: false if there are too many items
inline bool grid_of(const Batch& b, int own, int Hkv, int per, Grid& q, dim3& grid) {
  const int64_t tiles = b.T > 0 ? (b.T + own - 1) / own : 1;   // (T = 0: the slots are padding)
  const int64_t most = b.rows / own + b.N;                     // pairs that packed slots can have
  q.listed = b.off && b.N <= kListed && 2 * most < b.N * tiles;
  const int64_t items = q.listed ? most : b.N * tiles;
  if (items > 0x3fffffff || tiles > 0x3fffffff) return false;
  q.class_bits = Hkv % 8 == 0 ? 3 : (Hkv % 4 == 0 ? 2 : (Hkv % 2 == 0 ? 1 : 0));
  q.per = divisor((unsigned)per);
  q.N = divisor((unsigned)(b.N > 0 ? b.N : 1));
  q.items = (int)items;
  q.tiles = (int)tiles;
  q.own = own;
  const int64_t xcds = 8 >> q.class_bits, share = (items + xcds - 1) / xcds, y = share < 32768 ? share : 32768;
  grid = dim3((unsigned)((Hkv * 8 >> q.class_bits) * per), (unsigned)y, (unsigned)((share + y - 1) / y));
  return true;
}

// Whether tiles of 128 rows of Hq heads leave half of the CUs idle, and sequences span
// several.  (Forward: one sequence of 3488 tokens, 3 heads of 128, 84 tiles, 59 us with
// 128 rows a workgroup and 30 with 32 whose keys four waves share; 2 of 4096, 2 heads,
// 128 tiles, 70 and 43; 5 of 489, 12 heads, 240 tiles, 14 and 28.)
inline bool few_tiles(const Batch& b, int Hq) {
  const int64_t tiles = (b.T + kRows - 1) / kRows, packed = (b.rows + kRows - 1) / kRows;
  return tiles > 1 && (b.off ? (packed > b.N ? packed : b.N) : b.N * tiles) * Hq <= 128;
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// host side: the checks that the two calls share
inline bool good_rows(const void* p, int64_t ld, int64_t H, int64_t D, int64_t rows) {
  if (rows == 0) return true;
  return p && aligned16(p) && ld >= H * D && ld % 8 == 0 && ld <= (1 << 24);
}
inline dr_status check_batch(int64_t rows, int64_t N, int64_t T, const int32_t* off, int Hq, int Hkv, int64_t D,
                             dr_dtype dtype, float scale) {
  if (dtype != DR_BF16) return dtype == DR_F32 ? DR_ERR_UNSUPPORTED : DR_ERR_DTYPE;
  if (rows < 0 || N < 0 || T < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv || D < 1) return DR_ERR_ARG;
  if (!(scale > 0.f && scale < 1e30f)) return DR_ERR_ARG;
  if (N > 0x7fffffff || rows > 0x7fffffff || T > 0x7fffffff) return DR_ERR_UNSUPPORTED;
  if (!off && rows != N * T) return DR_ERR_ARG;
  if (off && N == 0 && rows > 0) return DR_ERR_ARG;
  if (Hq > 65536 || (D != 64 && D != 128)) return DR_ERR_UNSUPPORTED;
  return DR_OK;
}

}  // namespace attn
}  // namespace dr

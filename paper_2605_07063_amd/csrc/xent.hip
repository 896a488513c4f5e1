// Softmax cross entropy over a large vocabulary (dr_cross_entropy) and its
// gradient, without ever keeping the logits.
//
//   z = h W^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_{i, t_i};
//   dz_iv = g_i (exp(z_iv - lse_i) - [v = t_i]),  dh = dz W,  dW = dz^T h.
//
// All three products run on 256 x 256 tiles of bf16 MFMA with fp32
// accumulation (tile256.h).  Tokens without a loss are dropped first: the rows
// of h that count are copied next to each other, so that no product spends time
// on the others and nothing of theirs (NaN included) enters a sum.
// Forward: a tile of logits is reduced where it stands to each row's maximum
// and sum of exponentials over the tile's columns; a second kernel joins the
// tiles' pairs.  Backward: the logits are formed again, a piece of the
// vocabulary at a time; dz of the piece is kept in bf16 (one rounding; see
// significand()), multiplied with the piece of W into fp32 sums of dh, and with h
// into the piece's rows of dW.
#include "tile256.h"

namespace dr {
namespace xent {
namespace {

constexpr int kT = kTileRows;          // output tile edge
constexpr int kCols = kTileStepCols;   // reduction indices per step
constexpr int64_t kPieceBytes = (int64_t)512 << 20;   // dz of a piece, and
constexpr int64_t kPieceMin = 8192;                   // vocabulary entries of one at least
constexpr int64_t kPieceMax = 1 << 22;                // and at most (a panel spans less than 4 GiB)
constexpr int64_t kCUs = 256;

// ---- tokens that carry a loss

constexpr int kPlanThreads = 1024, kPlanRows = 8;   // rows of a thread: 1024 apart, read together

// list[0 .. count) = the rows with a target in [0, V), in order; and 1 beside the count
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const int* target, int M, int V, int* count, int* list) {
  constexpr int kWaves = kPlanThreads / 64;
  __shared__ __attribute__((aligned(16))) int part[kPlanRows][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int base = 0;
  for (long long r0 = tid; r0 - tid < M; r0 += kPlanThreads * kPlanRows) {
    int t[kPlanRows];
#pragma unroll
    for (int j = 0; j < kPlanRows; ++j) t[j] = r0 + j * kPlanThreads < M ? target[r0 + j * kPlanThreads] : -1;
    unsigned long long live[kPlanRows];
#pragma unroll
    for (int j = 0; j < kPlanRows; ++j) {
      live[j] = __ballot(t[j] >= 0 && t[j] < V);
      if (lane == 0) part[j][w] = __popcll(live[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPlanRows; ++j) {
      int at = base;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const int n = part[j][i];
        at += i < w ? n : 0;
        base += n;
      }
      if (live[j] >> lane & 1) list[at + __popcll(live[j] & ((1ull << lane) - 1))] = (int)(r0 + j * kPlanThreads);
    }
    __syncthreads();
  }
  if (tid == 0) count[0] = base, count[1] = __float_as_int(1.f);
}

// A token's g is split into its significand (in [1, 2)) and the rest, its sign and power
// of two.  dz is formed and rounded with the rest only, so that the target's entry, most
// of a row of dz, is close to a power of two and its rounding, which a whole row of dh or
// dW would share, nearly 0; the significand goes into dh after its sums, and into dW by
// way of h: its rows times their significand over the first token's (rounded, exact where
// all g are alike, as in a mean loss), and the sums times that one.  Where h is rounded so
// anyway, 1 - p of the target goes the same way: dz is formed over it, which makes the
// target's entry the power of two itself.  Errors against fp64, where rounding the
// outputs alone makes 1.66e-3 and rounding g dz made 2.1e-3 to 2.3e-3: one g for all, dh
// and dW 1.7e-3 to 1.8e-3; g of their own, dh 1.7e-3, dW 2.3e-3 to 2.4e-3 (2120 tokens,
// 154 entries: with 1 - p left in dz dh 1.95e-3, dW 2.57e-3), so that dW, which then takes
// the rounding of h in place of that of dz, gains nothing, and dh does.
__device__ __forceinline__ float significand(float g) {
  const unsigned u = __float_as_uint(g), e = u >> 23 & 0xff;
  return e == 0 || e == 255 ? 1.f : __uint_as_float((u & 0x7fffff) | 0x3f800000);
}
__device__ __forceinline__ float power(float g) {   // g = significand(g) * power(g)
  const unsigned u = __float_as_uint(g), e = u >> 23 & 0xff;
  return e == 0 || e == 255 ? g : __uint_as_float(u & 0xff800000);
}

// Row b: hc[b] = h[list[b]] if b < count; and if row b carries no loss, zeros
// in its outputs (those that are not NULL).
struct GatherArgs {
  const unsigned char* h;
  unsigned char *hc, *dh;
  unsigned char* hr;     // for the backward, the rows times their part of g
  const float* g;
  long long ldh, lddh;   // bytes
  const int* target;
  int *count, *list;
  float *loss, *lse;
  int M, V, D;
  // backward
  const unsigned char* W;
  long long ldw;         // bytes
  const float* row_lse;
  float* rest;           // [M]: what of a token's dz, beside the significand, goes by way of h
};
// 1 - p of row src's target, by the whole workgroup; 1 where that is less than 2^-7.  This p
// and the one that dz is formed from differ by fp32's roundings of the logit and of lse, about
// 2^-24 of their size: by 2^-20 for an lse of 12, 2^-13 of 1 - p at most, and by more in
// proportion for larger ones.  The target's entry of dz is the power of two only up to that;
// what divides dz multiplies dh and h again, so nothing else rests on it.
__device__ __forceinline__ float rest_of(const GatherArgs& a, long long src) {
  __shared__ float part[4];
  const unsigned char *h = a.h + src * a.ldh, *w = a.W + (long long)a.target[src] * a.ldw;
  float dot = 0.f;
  for (int c = threadIdx.x * 16; c < 2 * a.D; c += 256 * 16) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(h + c), y = *reinterpret_cast<const u32x4*>(w + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dot = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), dot);
      dot = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), dot);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) dot += __shfl_xor(dot, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
  __syncthreads();
  const float u = 1.f - __expf(part[0] + part[1] + part[2] + part[3] - a.row_lse[src]);
  return u > 0x1p-7f ? u : 1.f;   // (NaN: 1)
}
// row src of h to row dst of hc, and of hr, given the first token that counts
__device__ __forceinline__ void copy_row(const GatherArgs& a, long long src, long long dst, int first) {
  const unsigned char* h = a.h + src * a.ldh;
  float f = 1.f;
  if (a.g) {   // (the same for the whole workgroup)
    f = significand(a.g[src]) / significand(a.g[first]);
    const float u = f == 1.f ? 1.f : rest_of(a, src);
    f *= u;
    if (threadIdx.x == 0) a.rest[dst] = u;
  }
  for (int c = threadIdx.x * 16; c < 2 * a.D; c += 256 * 16) {
    u32x4 v = *reinterpret_cast<const u32x4*>(h + c);
    *reinterpret_cast<u32x4*>(a.hc + dst * (2ll * a.D) + c) = v;
    if (!a.hr) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = pack_bf16(__uint_as_float(v[e] << 16) * f, __uint_as_float(v[e] & 0xffff0000u) * f);
    *reinterpret_cast<u32x4*>(a.hr + dst * (2ll * a.D) + c) = v;
  }
}
__device__ __forceinline__ void no_loss(const GatherArgs& a, long long b) {
  if (a.dh)
    for (int c = threadIdx.x * 16; c < 2 * a.D; c += 256 * 16)
      *reinterpret_cast<u32x4*>(a.dh + b * a.lddh + c) = u32x4{0u, 0u, 0u, 0u};
  if (threadIdx.x == 0) {
    if (a.loss) a.loss[b] = 0.f;
    if (a.lse) a.lse[b] = 0.f;
  }
}
__global__ __launch_bounds__(256) void gather_kernel(GatherArgs a) {
  const long long b = blockIdx.x;
  if (b < *a.count) copy_row(a, a.list[b], b, a.list[0]);
  if (a.g && b == 0 && threadIdx.x == 0 && *a.count > 0) a.count[1] = __float_as_int(significand(a.g[a.list[0]]));
  const int t = a.target[b];
  if (t < 0 || t >= a.V) no_loss(a, b);
}
// Both in one launch for few tokens: every block counts the targets before its row
// (2048 rows: 16 MB of reads from L2 in all, less than a launch costs).
constexpr int64_t kCountAll = 2048;
__global__ __launch_bounds__(256) void count_gather_kernel(GatherArgs a) {
  __shared__ int part[3][4];
  const int b = blockIdx.x, tid = threadIdx.x;
  int before = 0, total = 0, first = 0x7fffffff;
#pragma unroll 8
  for (int r = tid; r < a.M; r += 256) {
    const int t = a.target[r], live = t >= 0 && t < a.V;
    total += live;
    before += r < b ? live : 0;
    first = live && r < first ? r : first;
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    before += __shfl_xor(before, o, 64);
    total += __shfl_xor(total, o, 64);
    const int x = __shfl_xor(first, o, 64);
    first = x < first ? x : first;
  }
  if ((tid & 63) == 0) part[0][tid >> 6] = before, part[1][tid >> 6] = total, part[2][tid >> 6] = first;
  __syncthreads();
  before = part[0][0] + part[0][1] + part[0][2] + part[0][3];
#pragma unroll
  for (int i = 0; i < 4; ++i) first = part[2][i] < first ? part[2][i] : first;
  if (b == 0 && tid == 0) {
    a.count[0] = part[1][0] + part[1][1] + part[1][2] + part[1][3];
    a.count[1] = __float_as_int(a.g && first < a.M ? significand(a.g[first]) : 1.f);
  }
  const int t = a.target[b];
  if (t < 0 || t >= a.V) {
    no_loss(a, b);
    return;
  }
  if (tid == 0) a.list[before] = b;
  copy_row(a, b, before, first);
}

// ---- operands of a tile product

// By rows: entry (r, k) at base + r ld + 2 k, `lines` rows (the tile's own) of
// k_end columns.  By lines: entry (k, c) at base + k ld + 2 c, `lines` columns,
// k_end rows; read through the transposing LDS read.  Entries outside read as 0.
struct Operand {
  const unsigned char* base;
  long long ld;
  int lines, k_end;
};

// A panel of LINES (256 or 64) lines by 64 reduction indices in LDS.  By rows: 16-row
// blocks of 2 KB (swz_read).  By lines: 64 token rows of 2 LINES bytes, in 32-byte
// slots of 16 lines; a transposing read takes 4 token rows of one slot, and the
// slots of the eight rows that 32 lanes touch (q = r & 3, bit 3 of r) are permuted
// so that they cover all banks: over eight slots of a 512-byte row, or over four
// and the two halves of a 256-byte pair of rows.
template <bool BY_ROWS, int LINES = kT>
struct Loader {
  static constexpr int kDma = LINES / 32;                     // instructions of a wave per step
  static constexpr int kRowsPer = LINES == kT ? 2 : 8;        // by lines: token rows of one
  static __device__ __forceinline__ int slot(int r) {
    return LINES == kT ? slot_xor(r) : (((r >> 1) & 1) | (((r >> 3) & 1) << 1));
  }
  const unsigned char* base;
  unsigned off[kDma];   // by rows: this lane's rows; by lines: this lane's columns; or kOobOffset
  unsigned ld;
  int r0, k_end;
  unsigned rbase;
  int fx;
  // first: the wave's first 16-line block
  __device__ __forceinline__ void init(const Operand& o, int w, int lane, int first) {
    base = o.base;
    k_end = o.k_end;
    ld = (unsigned)o.ld;
    if constexpr (BY_ROWS) {
#pragma unroll
      for (int u = 0; u < kDma; ++u) {
        const int r = 8 * (w + 4 * u) + (lane >> 3);
        off[u] = r < o.lines ? (unsigned)r * ld : kOobOffset;
      }
      r0 = w;   // half blocks w + 4 u: their parity is w's
      rbase = (unsigned)first * 2048;
    } else {
      constexpr int kLanes = 64 / kRowsPer;   // of a row
      r0 = kRowsPer * w + lane / kLanes;
#pragma unroll
      for (int u = 0; u < kDma; ++u) {
        if (u > 1 && LINES == kT) {   // (the permutation repeats)
          off[u] = off[u & 1];
          continue;
        }
        const int col = 16 * (((lane % kLanes) >> 1) ^ slot(r0 + 4 * kRowsPer * u)) + 8 * (lane & 1);
        off[u] = col < o.lines ? (unsigned)col * 2 : kOobOffset;
      }
      const int g = lane >> 4, tq = (lane >> 2) & 3;
      fx = first ^ slot(8 * g + tq);
      rbase = (unsigned)((8 * g + tq) * (2 * LINES) + (lane & 3) * 8);
    }
  }
  // DMA u < kDma of step t into the panel at LDS offset dst
  __device__ __forceinline__ void dma(int t, int u, unsigned dst, int w, int lane) const {
    unsigned v;
    const unsigned char* b = base;
    if constexpr (BY_ROWS) {
      const int col = t * kCols + 8 * swz_seg_of_lane(lane, r0 & 1);
      v = off[u] == kOobOffset || col >= k_end ? kOobOffset : off[u] + (unsigned)col * 2;
    } else {
      const int r = r0 + 4 * kRowsPer * u;
      b += (long long)t * kCols * ld;
      v = off[u] == kOobOffset || t * kCols + r >= k_end ? kOobOffset : off[u] + (unsigned)r * ld;
    }
    dma16_untracked(b, dst + (w + 4 * u) * 1024, v);
  }
  // fragment of 16-line block b, 32-index half kh
  __device__ __forceinline__ u32x4 frag(const unsigned char* panel, int b, int kh, int lane) const {
    if constexpr (BY_ROWS) {
      return swz_read(panel + rbase + b * 2048, lane & 15, 4 * kh + (lane >> 4));
    } else {
      const unsigned char* p = panel + kh * (32 * 2 * LINES) + rbase + (unsigned)((fx ^ b) * 32);
      const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr16(p));
      const uint2 hi = __builtin_bit_cast(uint2, lds_read_tr16(p + 4 * 2 * LINES));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
};

// acc[i][j]: lines 16 i of A's half by lines 16 j of B's half of this wave.  Lane l
// holds line l % 16 of B's block j, and in its four registers lines 4 (l / 16) .. + 3
// of A's block i: with the output's columns as A and its rows as B, four values
// that stand next to each other.
template <bool A_ROWS, bool B_ROWS>
__device__ __forceinline__ void product(unsigned char* lds, const Operand& A, const Operand& B, int k_end, f32x4 (&acc)[8][8]) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Loader<A_ROWS> la;
  Loader<B_ROWS> lb;
  la.init(A, w, lane, 8 * (w >> 1));
  lb.init(B, w, lane, 8 * (w & 1));
  const unsigned lds0 = lds_offset(lds);
  auto dma1 = [&](int t, int st, int q) __attribute__((always_inline)) {
    const unsigned sb = lds0 + st * kTileStage;
    if (q & 1) lb.dma(t, q >> 1, sb + kTilePanel, w, lane);
    else la.dma(t, q >> 1, sb, w, lane);
  };
  auto rd1 = [&](u32x4* fa, u32x4* fb, const unsigned char* sa, int kh, int q) __attribute__((always_inline)) {
    if (q & 1) fb[q >> 1] = lb.frag(sa + kTilePanel, q >> 1, kh, lane);
    else fa[q >> 1] = la.frag(sa, q >> 1, kh, lane);
  };
  tile256_clear(acc);
  tile256_loop(lds, (k_end + kCols - 1) / kCols, dma1, rd1, acc);
  DR_WAIT_VM(0);
}

// Tile (ia, ib) of workgroup `id`, which runs on XCD id % 8.  The tiles have one
// order: groups of columns, in a group bands of at most 8 tile rows, in a band by
// columns; 32 tiles that follow each other are about h rows by 32 / h columns, and
// an XCD takes whole runs of 32, whose panels its L2 then holds.  The bands are as
// even as the rows allow and no run has a gap, since the rows of the tokens that
// count are known here only (2467 of 4111 tokens, 50257 entries, D = 2048: forward
// 0.72 ms with gaps in the last band's runs, 0.47 without).  With fewer than four
// tiles for a CU plain order.  The grid is made for the most tiles there can be;
// false past the last one.
__device__ __forceinline__ bool locate(int id, int ta, int tb, int& ia, int& ib) {
  const int n = ta * tb;
  if (n < 4 * (int)kCUs) {
    if (id >= n) return false;
    ia = id % ta;
    ib = id / ta;
    return true;
  }
  const int sl = id >> 3, at = (((sl >> 5) * 8 + (id & 7)) << 5) + (sl & 31);
  if (at >= n) return false;
  const int bands = (ta + 7) / 8, h = (ta + bands - 1) / bands, cw = 32 / h;
  const int group = at / (ta * cw), c0 = group * cw, in = at - c0 * ta;
  const int w = tb - c0 < cw ? tb - c0 : cw, band = in / (h * w), r0 = band * h;
  const int rows = ta - r0 < h ? ta - r0 : h, of = in - r0 * w;
  ib = c0 + of / rows;
  ia = r0 + of % rows;
  return true;
}
int grid_of(int64_t ta, int64_t tb) { return (int)((ta * tb + 255) / 256 * 256); }

struct Args {
  const unsigned char *hc, *W;   // hc: rows of the tokens that count, D columns
  const unsigned char* hr;       // the same times their part of g
  const float* rest;             // what else of a token's dz that part holds
  long long ldw;                 // bytes
  const int *target, *count, *list;
  int V, D, tb;
  // forward
  const unsigned char* h;        // all tokens' rows
  long long ldh;                 // bytes
  float2* part;                  // [parts][M]: maximum and sum of 128 columns (64 or 32 of a strip)
  int parts;
  long long M;
  // backward
  const float *lse, *g;
  unsigned char* dz;             // [M][ldz] bf16, the piece's columns v0 .. v1 - 1
  long long ldz;                 // bytes
  int v0, v1;
  float* sum;                    // [splits][M][D]: dh's sums
  int splits, first;
  unsigned char *dh, *dW;
  long long lddh, lddw;          // bytes
  float* wsum;                   // [wsplits][v1 - v0][D]: dW's sums over parts of the tokens
  int wsplits;
};

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ Operand tokens_by_rows(const Args& a, int row0, int rows, int count) {
  return Operand{a.hc + (long long)row0 * (2ll * a.D), 2ll * a.D, count - row0 < rows ? count - row0 : rows, a.D};
}
// entries v0 + ib cols .. of the vocabulary, up to v1
__device__ __forceinline__ Operand vocabulary_by_rows(const Args& a, int ib, int cols) {
  const int c0 = a.v0 + ib * cols;
  return Operand{a.W + (long long)c0 * a.ldw, a.ldw, a.v1 - c0 < cols ? a.v1 - c0 : cols, a.D};
}
// columns ib cols .. of hr, of `count` tokens; ib kT .. of W, of entries v0 + k0 .. + n - 1
__device__ __forceinline__ Operand hidden_by_lines(const Args& a, int ib, int cols, int count) {
  return Operand{a.hr + 2ll * ib * cols, 2ll * a.D, a.D - ib * cols < cols ? a.D - ib * cols : cols, count};
}
__device__ __forceinline__ Operand weights_by_lines(const Args& a, int ib, int k0, int n) {
  return Operand{a.W + (long long)(a.v0 + k0) * a.ldw + 2ll * ib * kT, a.ldw, a.D - ib * kT < kT ? a.D - ib * kT : kT, n};
}
// dz has zeros from the last entry to the end of its 64 columns at least
__device__ __forceinline__ Operand dz_by_rows(const Args& a, int row0, int rows, int count, int k0, int n) {
  return Operand{a.dz + (long long)row0 * a.ldz + 2ll * k0, a.ldz, count - row0 < rows ? count - row0 : rows, (n + 7) / 8 * 8};
}
__device__ __forceinline__ Operand dz_by_lines(const Args& a, int ia, int lines, int count) {
  return Operand{a.dz + 2ll * ia * lines, a.ldz, lines, count};
}
// the part of the piece's entries that split takes: k0 .. k0 + the result - 1
__device__ __forceinline__ int split_range(const Args& a, int split, int splits, int& k0) {
  const int n = a.v1 - a.v0, steps = (n + kCols - 1) / kCols;
  k0 = (int)((long long)split * steps / splits) * kCols;
  const int k1 = (int)((long long)(split + 1) * steps / splits) * kCols;
  return (k1 < n ? k1 : n) - k0;
}
// Parts of a piece that dh's sums are taken over side by side, for tiles of
// `rows` tokens: as many as fill the CUs (the tokens that count are known here
// only; at most a.splits, whose sums the workspace holds).
__device__ __forceinline__ int splits_now(const Args& a, int count, int rows) {
  const int tiles = (count + rows - 1) / rows * a.tb;
  if (tiles == 0) return 0;
  const int s = (rows == kT ? 1 : 2) * (int)kCUs / tiles;
  return s < 1 ? 1 : (s < a.splits ? s : a.splits);
}

// The part of workgroup id, and its tile's number in it.  Those with work come first
// and without gaps: workgroups go to the shader engines in turn, so with gaps of
// empty ones one engine can get more than its CUs hold (80 tiles in 3 parts, each
// padded to 256 workgroups: 0.88 ms instead of 0.47).
__device__ __forceinline__ int part_of(int& id, int tiles, int splits) {
  if (splits <= 1) return 0;
  const int split = id / tiles;
  id -= split * tiles;
  return split;
}

// v of lanes l, l ^ 16, l ^ 32, l ^ 48 joined (without LDS: two exchanges of rows)
template <class F>
__device__ __forceinline__ float over_rows(float v, F&& f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// A token's maximum and sum of exponentials over what its four lanes (l % 16) hold:
// NI blocks of 16 columns, of which `left` from this lane's first on are in the
// vocabulary.  No column: 0 of -inf.
template <int NI>
__device__ __forceinline__ float2 token_stat(f32x4 (&x)[NI], int left) {
  float m = -INFINITY, s = 0.f;
  if (left < 16 * NI)
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * i + r >= left) x[i][r] = -INFINITY;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) m = fmaxf(m, x[i][r]);
  m = over_rows(m, [](float a, float b) { return fmaxf(a, b); });
  const float mc = (m == -INFINITY ? 0.f : m) * kLog2e;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f(x[i][r] * kLog2e - mc);
  return float2{m, over_rows(s, [](float a, float b) { return a + b; })};
}
// what dW's sums are multiplied by: the first token's significand, left beside the count
__device__ __forceinline__ float weight_scale(const Args& a) { return __int_as_float(a.count[1]); }
// a token's dz over the same columns: g (exp(z - lse) - [column = hit])
template <int NI>
__device__ __forceinline__ void token_dz(f32x4 (&x)[NI], int left, float lse2, float g, int hit) {
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) x[i][r] = __builtin_amdgcn_exp2f(x[i][r] * kLog2e - lse2);
  if (__any(hit >= 0 && hit < 16 * NI)) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (hit == 16 * i + r) x[i][r] -= 1.f;
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) x[i] *= g;
  if (left < 16 * NI)
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * i + r >= left) x[i][r] = 0.f;
}
__device__ __forceinline__ void store4(unsigned char* p, f32x4 v) {
  *reinterpret_cast<uint2*>(p) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}
// Blocks a and b of 16 columns each, as the lanes hold them, in bf16: lanes of odd
// and even rows of 16 exchange four columns, so that a lane stores 16 bytes and a
// store instruction 64 of each of its 16 rows (8 and 32 without: dW of 48 tokens, 128000
// entries, D = 4096, 1.05 GB: 372 us and 254).  This lane
// has eight columns from pair_col of the two blocks' 32.
__device__ __forceinline__ int pair_col(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }
__device__ __forceinline__ u32x4 pair_bf16(f32x4 a, f32x4 b) {
  const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(a[0], a[1]), pack_bf16(b[0], b[1]), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(a[2], a[3]), pack_bf16(b[2], b[3]), false, false);
  return u32x4{lo[0], hi[0], lo[1], hi[1]};
}

// Logits of 256 tokens by 256 entries: their statistics (DZ = false), or dz.  Bound by
// MFMA: 8192 tokens, 128000 entries, D = 4096 in 6.6 ms (1.30 PFLOP/s; MFMA busy 0.60 at
// 2.05 GHz), dz of 32768 of the entries in 1.85 ms (1.19); of a tile's 106 us 11 are its
// epilogue (54 of D = 2048).  Slower: 256 workgroups that take tile after tile, with the
// next one's first steps on their way meanwhile (111 us a tile, 58 of D = 2048).
template <bool DZ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void logit_kernel(Args a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTileRing];
  const int count = *a.count;
  int ia, ib;
  if (count == 0 || !locate(blockIdx.x, (count + kT - 1) / kT, a.tb, ia, ib)) return;
  const Operand A = vocabulary_by_rows(a, ib, kT), B = tokens_by_rows(a, ia * kT, kT, count);
  f32x4 acc[8][8];
  product<true, true>(lds, A, B, a.D, acc);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wc = w >> 1, wr = w & 1;
  const int col = 128 * wc + 4 * (lane >> 4), left = A.lines - col;   // this lane's first column
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int row = 128 * wr + 16 * j + (lane & 15);
    const bool in = row < B.lines;
    const long long at = (long long)ia * kT + row;
    f32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = acc[i][j];
    if constexpr (DZ) {
      const int src = in ? a.list[at] : 0;
      token_dz<8>(x, left, in ? a.lse[src] * kLog2e : 0.f, in ? power(a.g[src]) / a.rest[at] : 0.f,
                  in ? a.target[src] - a.v0 - ib * kT - col : -1);
      unsigned char* out = a.dz + at * a.ldz + 2ll * (ib * kT + 128 * wc + pair_col(lane));
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const u32x4 v = pair_bf16(x[i], x[i + 1]);
        if (in) *reinterpret_cast<u32x4*>(out + 32 * i) = v;
      }
    } else {
      const float2 st = token_stat<8>(x, left);
      if (lane < 16 && in) a.part[(2ll * ib + wc) * a.M + at] = st;
    }
  }
}

// sums of dh: += dz W over a part of the piece's vocabulary entries (8192 tokens,
// 32768 entries, D = 4096: 1.74 ms, 1.26 PFLOP/s)
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void dh_kernel(Args a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTileRing];
  const int count = *a.count, ta = (count + kT - 1) / kT, splits = splits_now(a, count, kT);
  int id = blockIdx.x, ia, ib, k0;
  const int split = part_of(id, ta * a.tb, splits);
  if (split >= splits || !locate(id, ta, a.tb, ia, ib)) return;
  const int n = split_range(a, split, splits, k0);
  const Operand A = weights_by_lines(a, ib, k0, n), B = dz_by_rows(a, ia * kT, kT, count, k0, n);
  f32x4 acc[8][8];
  product<false, true>(lds, A, B, n, acc);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = 128 * (w >> 1) + 4 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int row = 128 * (w & 1) + 16 * j + (lane & 15);
    if (row >= B.lines) continue;
    float* out = a.sum + (split * a.M + (long long)ia * kT + row) * a.D + ib * kT + col;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (col + 16 * i >= A.lines) continue;   // (D is a multiple of 8)
      f32x4 v = acc[i][j];
      if (!a.first) v += *reinterpret_cast<const f32x4*>(out + 16 * i);
      *reinterpret_cast<f32x4*>(out + 16 * i) = v;
    }
  }
}

// dh = the splits' sums in order, at the tokens' own rows: 1024 columns a block
__global__ __launch_bounds__(256) void dh_store_kernel(Args a, int rows) {
  const long long b = blockIdx.x;
  const int count = *a.count, splits = splits_now(a, count, rows);
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (b >= count || c >= a.D) return;
  const int row = a.list[b];
  float f = significand(a.g[row]) * a.rest[b];   // (ahead of the sums, which it would wait for otherwise)
  asm volatile("" : "+v"(f));
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(a.sum + (s * a.M + b) * a.D + c);
  store4(a.dh + (long long)row * a.lddh + 2 * c, v * f);
}

// the same of dW's parts
__global__ __launch_bounds__(256) void dw_store_kernel(Args a) {
  const long long b = blockIdx.x;
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (c >= a.D) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < a.wsplits; ++s)
    v += *reinterpret_cast<const f32x4*>(a.wsum + ((long long)s * (a.v1 - a.v0) + b) * a.D + c);
  store4(a.dW + (a.v0 + b) * a.lddw + 2 * c, v * weight_scale(a));
}

// rows v0 .. v1 - 1 of dW = dz^T h (the same sizes: 1.69 ms, 1.30 PFLOP/s)
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void dw_kernel(Args a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTileRing];
  const int count = *a.count;
  int ia, ib;
  if (!locate(blockIdx.x, (a.v1 - a.v0 + kT - 1) / kT, a.tb, ia, ib)) return;
  const Operand A = hidden_by_lines(a, ib, kT, count), B = dz_by_lines(a, ia, kT, count);
  f32x4 acc[8][8];
  product<false, false>(lds, A, B, count, acc);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = 128 * (w >> 1) + pair_col(lane);   // (D is a multiple of 8)
  const float scale = weight_scale(a);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int row = ia * kT + 128 * (w & 1) + 16 * j + (lane & 15);
    unsigned char* out = a.dW + (long long)(a.v0 + row) * a.lddw + 2ll * (ib * kT + col);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const u32x4 v = pair_bf16(acc[i][j] * scale, acc[i + 1][j] * scale);
      if (row < a.v1 - a.v0 && col + 16 * i < A.lines) *reinterpret_cast<u32x4*>(out + 32 * i) = v;
    }
  }
}

// ---- the same products in strips: 64 rows of the output by 256 or 64 columns
//
// For few tokens a tile of 256 would multiply mostly zeros, and one workgroup per CU
// does not keep enough of W under way; for small outputs tiles of 256 leave most CUs
// idle.  Two workgroups share a CU (four of 64 columns), each wave takes 64 columns (32
// by 32), and the operands go through two stages of 40 KB (16 KB).  For few tokens bound
// by reading W, or writing dW: 48 tokens, 128000 entries, D = 4096 (1.05 GB): statistics
// 175 us (6.0 TB/s), dz 180, dh 232, dW 225 to 283.
constexpr int kStrip = 64;
constexpr int kStripB = kStrip * kCols * 2;

// v of the lanes up to this one, added
__device__ __forceinline__ int sum_upto(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int x = __shfl_up(v, o, 64);
    if (lane >= o) v += x;
  }
  return v;
}
// N targets from row r on: which carry a loss (bit i: row r + i); none past M
template <int N>
__device__ __forceinline__ unsigned live_rows(const int* target, long long r, int M, int V) {
  int t[N];
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = r + i < M ? target[r + i] : -1;
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m |= t[i] >= 0 && t[i] < V ? 1u << i : 0u;
  return m;
}
// The tokens that count of M <= kCountAll, counted by the workgroup itself: returns how
// many there are, and leaves the rows of h of strip id % (strips that they make) in own.
// The first workgroup of a strip leaves its part of the list (and workgroup 0 the count,
// and zeros where there is no loss) for the kernel that joins the parts.
__device__ __forceinline__ int own_rows(const Args& a, int id, int* own, int* count, int* list, float* loss, float* lse) {
  constexpr int kOwn = (int)kCountAll / 256;   // rows of a thread at most
  const int tid = threadIdx.x, lane = tid & 63, per = ((int)a.M + 255) / 256;
  int* waves = own + kStrip;
  const int r0 = tid * per, end = r0 + per < a.M ? r0 + per : (int)a.M;
  const unsigned live = live_rows<kOwn>(a.target, r0, end, a.V);
  const int n = __popc(live), upto = sum_upto(n, lane);
  if (lane == 63) waves[tid >> 6] = upto;
  __syncthreads();
  int at = upto - n, total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at += i < tid >> 6 ? waves[i] : 0;
    total += waves[i];
  }
  const int strips = (total + kStrip - 1) / kStrip, first = (strips ? id % strips : 0) * kStrip;
  at -= first;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int r = r0 + i;
    if (live >> i & 1) {
      if (at >= 0 && at < kStrip) {
        own[at] = r;
        if (id < strips) list[first + at] = r;
      }
      ++at;
    } else if (id == 0 && r < end) {
      loss[r] = 0.f;
      lse[r] = 0.f;
    }
  }
  if (id == 0 && tid == 0) *count = total;
  __syncthreads();
  return total;
}

enum { kStat, kDz, kDh, kDw, kDwPart };   // (the last: fp32 sums over a part of the tokens)
// OWN (kStat): counts its tokens itself and reads their rows of h; grid of all strips
// that M tokens can have
template <int MODE, int COLS, bool OWN = false>
__global__ __launch_bounds__(256, COLS == kT ? 2 : 4) void strip_kernel(Args a, int* own_count = nullptr,
                                                                        int* own_list = nullptr, float* loss = nullptr,
                                                                        float* lse = nullptr) {
  constexpr int kRowWaves = COLS == kT ? 1 : 2, kColWaves = 4 / kRowWaves;   // a wave's place in the output
  constexpr int NI = COLS / 16 / kColWaves, NJ = kStrip / 16 / kRowWaves;    // its blocks of columns, rows
  constexpr int kPanel = COLS * kCols * 2, kStage = kPanel + kStripB;
  constexpr bool kOfW = MODE == kDw || MODE == kDwPart;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * kStage];
  int count;
  if constexpr (OWN) count = own_rows(a, blockIdx.x, reinterpret_cast<int*>(lds), own_count, own_list, loss, lse);
  else count = *a.count;
  // strips of the output; those of one panel of columns follow each other
  const int ta = ((kOfW ? a.v1 - a.v0 : count) + kStrip - 1) / kStrip;
  if (ta == 0) return;
  int id = blockIdx.x;
  const int splits = MODE == kDh ? splits_now(a, count, kStrip) : (MODE == kDwPart ? a.wsplits : 1);
  const int split = part_of(id, ta * a.tb, splits);
  const int ia = id % ta, ib = id / ta;
  if (ib >= a.tb || split >= splits) return;
  Operand A, B;   // the output's columns, rows
  int k_end = a.D;
  if constexpr (MODE == kDh) {
    int k0;
    k_end = split_range(a, split, splits, k0);
    A = weights_by_lines(a, ib, k0, k_end);
    B = dz_by_rows(a, ia * kStrip, kStrip, count, k0, k_end);
  } else if constexpr (MODE == kDw) {
    k_end = count;
    A = hidden_by_lines(a, ib, COLS, count);
    B = dz_by_lines(a, ia, kStrip, count);
  } else if constexpr (MODE == kDwPart) {
    const int n = (count + kCols - 1) / kCols, k0 = split * n / splits * kCols, k1 = (split + 1) * n / splits * kCols;
    k_end = __builtin_amdgcn_readfirstlane((k1 < count ? k1 : count) - k0);
    A = hidden_by_lines(a, ib, COLS, k_end);
    B = dz_by_lines(a, ia, kStrip, k_end);
    A.base += __builtin_amdgcn_readfirstlane(k0) * A.ld;
    B.base += __builtin_amdgcn_readfirstlane(k0) * B.ld;
  } else {
    A = vocabulary_by_rows(a, ib, COLS);
    B = tokens_by_rows(a, ia * kStrip, kStrip, count);
  }
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wc = w / kRowWaves, wr = w % kRowWaves;
  Loader<MODE == kStat || MODE == kDz, COLS> la;
  Loader<!kOfW, kStrip> lb;
  la.init(A, w, lane, NI * wc);
  lb.init(B, w, lane, NJ * wr);
  if constexpr (OWN) {
    lb.base = a.h;
#pragma unroll
    for (int u = 0; u < Loader<true, kStrip>::kDma; ++u) {
      const int r = 8 * (w + 4 * u) + (lane >> 3);
      if (r < B.lines) lb.off[u] = (unsigned)reinterpret_cast<const int*>(lds)[r] * (unsigned)a.ldh;
    }
    __syncthreads();   // (the rows' numbers stand where the operands go)
  }
  const unsigned lds0 = lds_offset(lds);
  const int steps = (k_end + kCols - 1) / kCols;
  // Along W's rows the wide strips start at different steps: with all at the same columns
  // of rows 8 KB apart they wait for the same memory channels (48 tokens, 128000 entries,
  // D = 4096: 197 to 255 us, by where W lies, and 185).  Narrow ones, whose strips share
  // what L2 holds of W and h, lose by it (167 tokens, 9750 entries, D = 4016: 49 and 55).
  const int start = COLS == kT && (MODE == kStat || MODE == kDz) && steps > 0 ? ib % steps : 0;
  auto load = [&](int t) {
    const unsigned st = lds0 + (t & 1) * kStage;
    const int k = t + start < steps ? t + start : t + start - steps;
#pragma unroll
    for (int u = 0; u < kStrip / 32; ++u) lb.dma(k, u, st + kPanel, w, lane);
#pragma unroll
    for (int u = 0; u < COLS / 32; ++u) la.dma(k, u, st, w, lane);
  };
  f32x4 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  load(0);
  for (int t = 0; t < steps; ++t) {
    DR_WAIT_VM(0);
    DR_LDS_SYNC();
    if (t + 1 < steps) load(t + 1);
    const unsigned char* sa = lds + (t & 1) * kStage;
    u32x4 fa[2][NI], fb[2][NJ];
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) fb[kh][j] = lb.frag(sa + kPanel, j, kh, lane);
#pragma unroll
      for (int i = 0; i < NI; ++i) fa[kh][i] = la.frag(sa, i, kh, lane);
    }
    __builtin_amdgcn_sched_barrier(0);   // (the compiler otherwise waits four times for a few reads)
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = mma_bf16(fa[kh][i], fb[kh][j], acc[i][j]);
  }
  DR_WAIT_VM(0);
  const int col = 16 * NI * wc + 4 * (lane >> 4), left = A.lines - col;   // this lane's first column
  const float scale = MODE == kDw ? weight_scale(a) : 1.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int row = 16 * (NJ * wr + j) + (lane & 15);
    const long long at = (long long)ia * kStrip + row;
    const bool in = kOfW ? at < a.v1 - a.v0 : row < B.lines;
    f32x4 x[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) x[i] = acc[i][j];
    if constexpr (MODE == kStat) {
      const float2 st = token_stat<NI>(x, left);
      if (lane < 16 && in) a.part[((long long)kColWaves * ib + wc) * a.M + at] = st;
    } else if constexpr (MODE == kDz) {
      const int src = in ? a.list[at] : 0;
      token_dz<NI>(x, left, in ? a.lse[src] * kLog2e : 0.f, in ? power(a.g[src]) / a.rest[at] : 0.f,
                  in ? a.target[src] - a.v0 - ib * COLS - col : -1);
      unsigned char* out = a.dz + at * a.ldz + 2ll * (ib * COLS + 16 * NI * wc + pair_col(lane));
#pragma unroll
      for (int i = 0; i < NI; i += 2) {
        const u32x4 v = pair_bf16(x[i], x[i + 1]);
        if (in) *reinterpret_cast<u32x4*>(out + 32 * i) = v;
      }
    } else if constexpr (MODE == kDh) {
      float* out = a.sum + (split * a.M + at) * a.D + ib * COLS + col;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (!in || 16 * i >= left) continue;
        if (!a.first) x[i] += *reinterpret_cast<const f32x4*>(out + 16 * i);
        *reinterpret_cast<f32x4*>(out + 16 * i) = x[i];
      }
    } else if constexpr (MODE == kDwPart) {
      float* out = a.wsum + ((long long)split * (a.v1 - a.v0) + at) * a.D + ib * COLS + col;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (in && 16 * i < left) *reinterpret_cast<f32x4*>(out + 16 * i) = x[i];
    } else {
      const int pair = 16 * NI * wc + pair_col(lane);
      unsigned char* out = a.dW + (a.v0 + at) * a.lddw + 2ll * (ib * COLS + pair);
#pragma unroll
      for (int i = 0; i < NI; i += 2) {
        const u32x4 v = pair_bf16(x[i] * scale, x[i + 1] * scale);
        if (in && pair + 16 * i < A.lines) *reinterpret_cast<u32x4*>(out + 32 * i) = v;
      }
    }
  }
}

// ROWS tokens a block of 1024 threads, which join each token's partial pairs; then a
// wave each takes the targets' logits as dot products.  16 tokens, or 2 where there
// are few tokens and many pairs of each.
constexpr int kJoinThreads = 1024;
// what a sum of exponentials relative to m counts relative to top >= m (a sum
// that has no column yet is 0 relative to -inf, and NaN stays NaN)
__device__ __forceinline__ float scale_to(float m, float top) { return m == -INFINITY ? 1.f : __expf(m - top); }
template <int ROWS>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(Args a, float* loss, float* lse) {
  constexpr int kRuns = kJoinThreads / ROWS;
  __shared__ float2 part[kJoinThreads];
  const int count = *a.count;
  const int j0 = blockIdx.x * ROWS;
  if (j0 >= count) return;
  const int r = threadIdx.x % ROWS, run = threadIdx.x / ROWS;
  float m = -INFINITY, s = 0.f;
  if (j0 + r < count) {
#pragma unroll 4
    for (int p = run; p < a.parts; p += kRuns) {
      const float2 v = a.part[(long long)p * a.M + j0 + r];
      const float top = fmaxf(m, v.x);
      s = s * scale_to(m, top) + v.y * scale_to(v.x, top);
      m = top;
    }
  }
  part[threadIdx.x] = float2{m, s};
  __syncthreads();
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;   // wave w: token j0 + w
  if (w >= ROWS || j0 + w >= count) return;
  m = -INFINITY, s = 0.f;
#pragma unroll
  for (int i = 0; i < kRuns / 64; ++i) {
    const float2 v = part[(i * 64 + lane) * ROWS + w];
    const float top = fmaxf(m, v.x);
    s = s * scale_to(m, top) + v.y * scale_to(v.x, top);
    m = top;
  }
  float top = m;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
  float total = s * scale_to(m, top);
  const int row = a.list[j0 + w];
  const unsigned char* hr = a.h + (long long)row * a.ldh;
  const unsigned char* wr = a.W + (long long)a.target[row] * a.ldw;
  float dot = 0.f;
#pragma unroll 4
  for (int c = lane * 16; c < 2 * a.D; c += 64 * 16) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(hr + c), y = *reinterpret_cast<const u32x4*>(wr + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dot = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), dot);
      dot = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), dot);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    total += __shfl_xor(total, o, 64);
    dot += __shfl_xor(dot, o, 64);
  }
  if (lane == 0) {
    const float l = top + __logf(total);
    lse[row] = l;
    loss[row] = l - dot;
  }
}

// ---- host side

int64_t tiles_of(int64_t n) { return (n + kT - 1) / kT; }
// vocabulary entries of a piece (a multiple of the tile)
int64_t piece_of(int64_t M, int64_t V) {
  int64_t p = kPieceBytes / (2 * M);
  if (p < kPieceMin) p = kPieceMin;
  if (p > kPieceMax) p = kPieceMax;
  if (p > V) p = V;
  return tiles_of(p) * kT;
}
// Strips where one holds all tokens, or where tiles of 256 of the rows x cols output,
// `splits` times over, would not fill half the CUs.  (D = 4096: 48 tokens, 128000
// entries, forward 185 us in strips and 277 in tiles; 128 tokens, 50257 entries, 132
// and 125; 640 tokens, D = 256, 1000 entries 17 and 22.)  dW, whose time is its
// writing then, takes strips up to 256 tokens (D = 4096, 128000 entries, backward: 256
// tokens 1.05 ms and 1.10, 512 tokens 1.73 and 1.71).
bool use_strips(int64_t M, int64_t rows, int64_t cols, int64_t splits = 1) {
  return M <= kStrip || tiles_of(rows) * tiles_of(cols) * splits < kCUs / 2;
}
int strips_of(int64_t n) { return (int)((n + kStrip - 1) / kStrip); }
// The logits' products (M tokens, n entries) also where there are few steps, and most of a
// tile's time is what its one workgroup a CU does before and after them.  (8192 tokens,
// 32768 entries: D = 64 forward 168 us in tiles and 124 in strips, backward 584 and 568; D
// = 128 190 and 151, 628 and 629; D = 256 233 and 203, 752 and 778.)
// Of many steps (above 512 dimensions) and few tokens only up to 9/8 strips a CU: the strips
// of one panel of W run on different XCDs, each of which reads it.  Forward, strips and tiles,
// us, D = 2048 | 4096: 256 tokens by 16344 entries (256 strips) 49 and 57 | 80 and 96, by 20440
// (320) 67 and 57 | 109 and 96; 512 by 8152 (256) 45 and 59 | 81 and 99, by 10200 (320) 62 and
// 58 | 110 and 99; 700 by 6616 (286) 54 and 59 | 97 and 100, by 10712 (462) 68 and 60 | 130 and
// 102.  Above 768 tokens, whose W is smaller for as many strips, as otherwise: 1000 by 7900
// (496 strips, 124 tiles) 59 and 60 | 105 and 104, 2048 by 2800 (352, 88) 51 and 60 | 86 and
// 104; and at D = 512: 256 by 20440 24 and 27, by 32216 (126 tiles) 31 and 28.
bool logit_strips(int64_t M, int64_t n, int64_t D) {
  if (D > 512 && M > kStrip && M <= 768) return strips_of(M) * tiles_of(n) <= kCUs + kCUs / 8;
  return use_strips(M, M, n) || D < 256;
}
// Strips of 64 x 64 where those of 64 x 256 would leave CUs idle: a CU's DMA brings
// 40 KB of operands a step of 64 indices in 0.6 us, however few workgroups there are.
// (248 tokens, 531 entries, D = 2256: forward 31 us with 256 columns and 18 with 64,
// backward 51 and 37; 167 tokens, 9750 entries, D = 4016: 71 and 49, 140 and 116; with
// 500 strips of 256, 48 tokens, 128000 entries, D = 4096, 191 and 239 before they started
// at different steps.)
// Strips of tokens, of which some may not count, up to twice as many (1003 tokens of
// which 200 count, 5217 entries, D = 2280: forward 45 us and 32, backward 89 and 73).
bool narrow(int64_t strips, int64_t cols, bool tokens) {
  return strips * tiles_of(cols) < (tokens && strips > 1 ? 2 * kCUs : kCUs);
}
// parts of a token's statistics (M tokens, V entries)
int64_t parts_of(int64_t M, int64_t V, int64_t D) {
  if (!logit_strips(M, V, D)) return 2 * tiles_of(V);
  return narrow(strips_of(M), V, true) ? 2 * strips_of(V) : 4 * tiles_of(V);
}
// most parts that dh's sums are taken over side by side: enough for a quarter of
// the tokens to fill the CUs, and 128 (976 tokens of which 195 count, 89197 entries,
// D = 184: backward 104 us, 138 with 32; 60 tokens, 50257 entries, D = 2048: 157 and 150)
int splits_of(int64_t M, int64_t V, int64_t D) {
  const int64_t steps = piece_of(M, V) / kCols;
  int64_t s = 4 * kCUs / (tiles_of(M) * tiles_of(D));
  if (s > 128) s = 128;
  if (s > steps / 4) s = steps / 4;
  return (int)(s < 1 ? 1 : s);
}
// Parts of the tokens that dW's sums are taken over where it is small and the tokens
// are many: enough for two workgroups a CU, of 256 tokens at least.  (7358
// tokens, 295 entries, D = 64: the whole backward 84 us, with 16 parts 40.)
int wsplits_of(int64_t M, int64_t V, int64_t D) {
  const int64_t rows = piece_of(M, V) < V ? piece_of(M, V) : V, n = (int64_t)strips_of(rows) * strips_of(D);
  if (n > 128 || M < 1024) return 1;
  int64_t s = 2 * kCUs / n;
  if (s > 16) s = 16;
  if (s > M / 256) s = M / 256;
  return (int)s;
}
struct Layout {
  size_t list, hc, hr, rest, part, dz, sum, wsum, end;
};
Layout layout(int64_t M, int64_t V, int64_t D, bool back) {
  Layout l;
  size_t at = 256;   // the count
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = align_up(at + bytes, 256);
    return here;
  };
  l.list = take((size_t)M * 4);
  l.hc = take((size_t)M * (size_t)D * 2);
  l.hr = l.rest = l.part = l.dz = l.sum = l.wsum = 0;
  if (back) {
    l.hr = take((size_t)M * (size_t)D * 2);
    l.rest = take((size_t)M * 4);
    l.dz = take((size_t)M * (size_t)piece_of(M, V) * 2);
    l.sum = take((size_t)splits_of(M, V, D) * (size_t)M * (size_t)D * 4);
    const int64_t ws = wsplits_of(M, V, D);
    if (ws > 1) l.wsum = take((size_t)ws * (size_t)(piece_of(M, V) < V ? piece_of(M, V) : V) * (size_t)D * 4);
  } else {
    l.part = take((size_t)parts_of(M, V, D) * (size_t)M * sizeof(float2));
  }
  l.end = at;
  return l;
}

template <int MODE, bool OWN = false, class... Rest>
void launch_strips(Args a, int64_t cols, int strips, hipStream_t hs, Rest... rest) {
  if (narrow(strips, cols, MODE != kDw)) {
    a.tb = strips_of(cols);
    strip_kernel<MODE, kStrip, OWN><<<strips * a.tb, 256, 0, hs>>>(a, rest...);
  } else {
    a.tb = (int)tiles_of(cols);
    strip_kernel<MODE, kT, OWN><<<strips * a.tb, 256, 0, hs>>>(a, rest...);
  }
}
void launch_gather(const GatherArgs& a, hipStream_t hs) {
  if (a.M > 0 && a.M <= kCountAll) {
    count_gather_kernel<<<a.M, 256, 0, hs>>>(a);
    return;
  }
  plan_kernel<<<1, kPlanThreads, 0, hs>>>(a.target, a.M, a.V, a.count, a.list);
  if (a.M > 0) gather_kernel<<<a.M, 256, 0, hs>>>(a);
}

bool sizes_ok(int64_t M, int64_t V, int64_t D) { return M >= 0 && V >= 1 && D >= 8 && D % 8 == 0; }
// A launch takes fewer than 2^32 threads per dimension: 2^24 workgroups of 256, those
// that grid_of adds among them.  (The gather has one a token.)
bool sizes_supported(int64_t M, int64_t V, int64_t D) {
  constexpr int64_t most = ((int64_t)1 << 24) - 1024;
  if (M >= (int64_t)1 << 24 || V > 0x7fffff00 || D > 65536) return false;
  const int64_t logits = (logit_strips(M, V, D) ? strips_of(M) : tiles_of(M)) * tiles_of(V);
  return logits <= most && strips_of(V) * tiles_of(D) <= most;
}
// W's rows are at most 2^22 values apart: a panel's 256 rows take 32-bit offsets.  Rows of
// the others are addressed one by one, in 64 bits.
constexpr int64_t kMaxLdw = 1 << 22, kMaxLd = (int64_t)1 << 32;
bool good(const void* p, int64_t ld, int64_t D, int64_t most = kMaxLd) {
  return p && aligned16(p) && ld >= D && ld % 8 == 0 && ld <= most;
}

}  // namespace
}  // namespace xent
}  // namespace dr

extern "C" size_t dr_cross_entropy_workspace_size(int64_t M, int64_t V, int64_t D, int backward) {
  using namespace dr::xent;
  if (M < 1 || !sizes_ok(M, V, D) || !sizes_supported(M, V, D)) return 0;
  return layout(M, V, D, backward != 0).end;
}

extern "C" dr_status dr_cross_entropy(const void* h, int64_t ldh, const void* W, int64_t ldw, const int32_t* target, int64_t M,
                                      int64_t V, int64_t D, dr_dtype dtype, float* loss, float* lse, void* workspace,
                                      size_t ws_bytes, void* stream) {
  using namespace dr;
  using namespace dr::xent;
  if (dtype != DR_BF16) return dtype == DR_F32 ? DR_ERR_UNSUPPORTED : DR_ERR_DTYPE;
  if (!sizes_ok(M, V, D)) return DR_ERR_ARG;
  if (M == 0) return DR_OK;
  if (!good(h, ldh, D) || !good(W, ldw, D, kMaxLdw) || !target || !loss || !lse) return DR_ERR_ARG;
  if (!sizes_supported(M, V, D)) return DR_ERR_UNSUPPORTED;
  const Layout l = layout(M, V, D, false);
  if (!workspace || ws_bytes < l.end) return DR_ERR_WORKSPACE;
  if (!aligned16(workspace)) return DR_ERR_ARG;
  unsigned char* ws = (unsigned char*)workspace;
  const hipStream_t hs = (hipStream_t)stream;
  int* count = (int*)ws;
  int* list = (int*)(ws + l.list);
  // (a workgroup counts for 3 us, which is less than the launch where there are few)
  const bool strips = logit_strips(M, V, D);
  const bool own = strips && M <= kCountAll && strips_of(M) * tiles_of(V) <= 4 * kCUs &&
                   (M * ldh + D) * 2 < (int64_t)kOobOffset;
  if (!own)
    launch_gather(GatherArgs{(const unsigned char*)h, ws + l.hc, nullptr, nullptr, nullptr, ldh * 2, 0, target, count, list,
                             loss, lse, (int)M, (int)V, (int)D},
                  hs);
  Args a = {};
  a.h = (const unsigned char*)h;
  a.ldh = ldh * 2;
  a.hc = ws + l.hc;
  a.W = (const unsigned char*)W;
  a.ldw = ldw * 2;
  a.target = target, a.count = count, a.list = list;
  a.V = (int)V, a.D = (int)D, a.M = M;
  a.part = (float2*)(ws + l.part);
  a.parts = (int)parts_of(M, V, D);
  a.tb = (int)tiles_of(V);
  a.v1 = (int)V;
  if (own) {
    launch_strips<kStat, true>(a, V, strips_of(M), hs, count, list, loss, lse);
  } else if (strips) {
    launch_strips<kStat>(a, V, strips_of(M), hs);
  } else {
    const int grid = grid_of(tiles_of(M), a.tb);
    logit_kernel<false><<<grid, 256, 0, hs>>>(a);
  }
  if (M <= 512 && a.parts > 64) join_kernel<2><<<(int)((M + 1) / 2), kJoinThreads, 0, hs>>>(a, loss, lse);
  else join_kernel<16><<<(int)((M + 15) / 16), kJoinThreads, 0, hs>>>(a, loss, lse);
  return launch_status();
}

extern "C" dr_status dr_cross_entropy_backward(const void* h, int64_t ldh, const void* W, int64_t ldw, const int32_t* target,
                                               const float* lse, const float* g, int64_t M, int64_t V, int64_t D,
                                               dr_dtype dtype, void* dh, int64_t lddh, void* dW, int64_t lddw, void* workspace,
                                               size_t ws_bytes, void* stream) {
  using namespace dr;
  using namespace dr::xent;
  if (dtype != DR_BF16) return dtype == DR_F32 ? DR_ERR_UNSUPPORTED : DR_ERR_DTYPE;
  if (!sizes_ok(M, V, D)) return DR_ERR_ARG;
  if ((dh && !good(dh, lddh, D)) || (dW && !good(dW, lddw, D))) return DR_ERR_ARG;
  if (M > 0 && (!good(h, ldh, D) || !good(W, ldw, D, kMaxLdw) || !target || !lse || !g)) return DR_ERR_ARG;
  if (!sizes_supported(M, V, D)) return DR_ERR_UNSUPPORTED;
  if (!dh && !dW) return DR_OK;
  if (M == 0 && !dW) return DR_OK;
  const int64_t rows = M > 0 ? M : 1;   // (no tokens: dW is written as zeros)
  const Layout l = layout(rows, V, D, true);
  if (!workspace || ws_bytes < l.end) return DR_ERR_WORKSPACE;
  if (!aligned16(workspace)) return DR_ERR_ARG;
  unsigned char* ws = (unsigned char*)workspace;
  const hipStream_t hs = (hipStream_t)stream;
  int* count = (int*)ws;
  int* list = (int*)(ws + l.list);
  launch_gather(GatherArgs{(const unsigned char*)h, ws + l.hc, (unsigned char*)dh, dW ? ws + l.hr : nullptr, g, ldh * 2,
                           lddh * 2, target, count, list, nullptr, nullptr, (int)M, (int)V, (int)D, (const unsigned char*)W,
                           ldw * 2, lse, (float*)(ws + l.rest)},
                hs);
  Args a = {};
  a.hc = ws + l.hc;
  a.hr = ws + l.hr;
  a.rest = (const float*)(ws + l.rest);
  a.W = (const unsigned char*)W;
  a.ldw = ldw * 2;
  a.target = target, a.count = count, a.list = list;
  a.V = (int)V, a.D = (int)D, a.M = rows;
  a.lse = lse, a.g = g;
  a.dz = ws + l.dz;
  const int64_t piece = piece_of(rows, V);
  a.ldz = piece * 2;
  a.sum = (float*)(ws + l.sum);
  a.splits = splits_of(rows, V, D);
  a.wsum = (float*)(ws + l.wsum);
  a.wsplits = wsplits_of(rows, V, D);
  a.dh = (unsigned char*)dh, a.lddh = lddh * 2;
  a.dW = (unsigned char*)dW, a.lddw = lddw * 2;
  const int64_t tm = tiles_of(rows), td = tiles_of(D);
  const bool strips = use_strips(M, M, D, a.splits);   // of dh
  for (int64_t v = 0; v < V; v += piece) {
    a.v0 = (int)v;
    a.v1 = (int)(v + piece < V ? v + piece : V);
    a.first = v == 0;
    const int64_t tv = tiles_of(a.v1 - a.v0);
    if (M > 0) {
      a.tb = (int)tv;
      if (logit_strips(M, a.v1 - a.v0, D)) {
        launch_strips<kDz>(a, a.v1 - a.v0, strips_of(M), hs);
      } else {
        const int grid = grid_of(tm, tv);
        logit_kernel<true><<<grid, 256, 0, hs>>>(a);
      }
    }
    a.tb = (int)td;
    if (dW) {
      if (a.wsplits > 1) {
        const int strips = strips_of(a.v1 - a.v0), panels = strips_of(D);
        a.tb = panels;
        strip_kernel<kDwPart, kStrip><<<strips * panels * a.wsplits, 256, 0, hs>>>(a);
        a.tb = (int)td;
        dw_store_kernel<<<dim3((int)(a.v1 - a.v0), (int)((D + 1023) / 1024)), 256, 0, hs>>>(a);
      } else if (M <= 256 || use_strips(M, a.v1 - a.v0, D)) {
        launch_strips<kDw>(a, D, strips_of(a.v1 - a.v0), hs);
      } else {
        const int grid = grid_of(tv, td);
        dw_kernel<<<grid, 256, 0, hs>>>(a);
      }
    }
    if (dh && M > 0) {
      if (strips) {
        const int most = strips_of(M) * a.tb, part = 2 * (int)kCUs;   // without parts, with them
        strip_kernel<kDh, kT><<<most > part ? most : part, 256, 0, hs>>>(a);
      } else {
        const int grid = grid_of(tm, td);
        dh_kernel<<<grid, 256, 0, hs>>>(a);
      }
    }
  }
  if (dh && M > 0) dh_store_kernel<<<dim3((int)M, (int)((D + 1023) / 1024)), 256, 0, hs>>>(a, strips ? kStrip : kT);
  return launch_status();
}

// Causal attention of a merged batch (dr_attention): packed or padded
// sequences, grouped heads, bf16 in and out.
//
//   S = scale Q K^T over the keys j <= i of row i's own sequence,
//   O = softmax(S) V,  lse = log sum exp S.
//
// A workgroup of four waves takes 128 query rows of one head, 32 a wave, and
// streams its keys and values through two LDS stages of 64 rows.  A wave forms
// S^T = K Q^T, so that a lane holds one query's scores: the softmax's running
// maximum and sum are a lane's own (its two halves join by one exchange), the
// scores go into O^T = V^T P^T as the B operand without leaving their lanes, and
// the rescaling of O is a product by a lane's own factor.  Scores, statistics
// and O are fp32; P is rounded to bf16 for its product with V, as V is.
//
// With D = 128 a SIMD holds two waves (204 registers), with D = 64 four; MFMA and
// softmax are about even (16 products and 128 VALU instructions, a quarter of them
// exponentials, for 32 rows by 64 keys of D = 64) and wait for each other.  32 query
// heads of 8 key heads, forward: 16 sequences of 1024, D = 128, 176 us (0.78 PFLOP/s;
// MFMA busy 0.39, VALU 0.41); 4 of 4096 550 us (1.00; MFMA busy 0.57 at the 1.58 GHz
// that power leaves); the same with D = 64 323 us (0.85; VALU busy 0.78); 72 examples of
// 128 to 512 tokens, D = 64, 93 us, of which Q, K, V and O of HBM take 59.  Slower:
// 64 rows a wave (D = 128 one wave a SIMD, +36 %; D = 64 +3 %), the values of a step beside
// the next one's scores (+11 to +14 %), half a step's scores beside the other half's
// weights (+15 to +23 %), raised priority around the products (no change).
#include "attn.h"

namespace dr {
namespace attn {
namespace {

constexpr int kStep = 64;   // rows of a streamed tile

struct FwdArgs {
  const unsigned char *q, *k, *v;
  unsigned char* o;
  float* lse;                          // [Hq][rows]
  long long ldq, ldk, ldv, ldo;        // bytes between rows
  Batch b;
  Grid grid;
  int Hq;
  float scale;
};

// Padding of the slot in a tile of OWN rows from q0 on: zeros, the last tile's workgroup
// to the slot's end.
template <int D, int OWN>
__device__ __forceinline__ void zero_padding(const FwdArgs& a, const Seq& s, int q0, bool last, int head, unsigned hb) {
  const long long from = q0 < s.len ? (s.len < q0 + OWN ? s.len : q0 + OWN) : q0;
  long long to = s.end - s.first;
  if (!last && q0 + OWN < to) to = q0 + OWN;
  if (from >= to) return;
  zero_rows<D * 2>(a.o + s.first * a.ldo + hb, a.ldo, from, to);
  for (long long r = from + threadIdx.x; r < to; r += kThreads) a.lse[(long long)head * a.b.rows + s.first + r] = 0.f;
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_kernel(FwdArgs a) {
  constexpr int kTile = kStep * D * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];   // two stages of K, V
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place at;
  if (!place_of(a.grid, a.b, at)) return;
  const int tile = at.place, head = at.khead * (int)a.grid.per.d + at.g;
  const Seq s = sequence(a.b, at.seq);
  const int q0 = tile * kRows;
  const unsigned hb = (unsigned)head * (D * 2), kb = (unsigned)at.khead * (D * 2);
  zero_padding<D, kRows>(a, s, q0, tile == at.tiles - 1, head, hb);
  if (q0 >= s.len) return;

  const unsigned char* kp = a.k + s.first * a.ldk + kb;
  const unsigned char* vp = a.v + s.first * a.ldv + kb;
  const unsigned ldk = (unsigned)a.ldk, ldv = (unsigned)a.ldv;
  TileLoad<D, kStep> lk, lv;
  lk.init(w, lane, ldk);
  lv.init(w, lane, ldv);
  const unsigned lds0 = lds_offset(lds);
  auto load = [&](int t) {
    const unsigned st = lds0 + (t & 1) * (2 * kTile);
    lk.issue(kp + (long long)t * kStep * ldk, s.len - t * kStep, ldk, st, w);
    lv.issue(vp + (long long)t * kStep * ldv, s.len - t * kStep, ldv, st + kTile, w);
  };
  // this wave's rows of Q into its quarter of the second stage, ahead of the first
  // step's keys: whole rows to an instruction.  (As fragments straight from memory
  // each would take 32 bytes of 32 rows.)
  const int qw = q0 + 32 * w, row = qw + (lane & 31);   // this wave's first row, this lane's
  {
    TileLoad<D, 32, 1> lq;
    lq.init(0, lane, (unsigned)a.ldq);
    lq.issue(a.q + (s.first + qw) * a.ldq + hb, s.len - qw, (unsigned)a.ldq, lds0 + 2 * kTile + w * (64 * D), 0);
  }
  load(0);
  TilePlace<D> place;
  place.init(lane);
  constexpr int kLoads = 2 * TileLoad<D, kStep>::kCount;   // of a step
  DR_WAIT_VM(kLoads);
  u32x4 qf[D / 16];
  tile_fragments<D>(lds + 2 * kTile + w * (64 * D), place, qf);
#pragma unroll
  for (int x = 0; x < D / 16; ++x) arrived(qf[x]);
  f32x16 o[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[cb][r] = 0.f;
  float m = -INFINITY, sum = 0.f;
  const float c = a.scale * kLog2e;
  // The reference m follows the running maximum only when that has passed it by
  // more than 8 powers of two: until then exponentials are at most 256, and O and
  // the sum need no rescaling, which is a product per value of O.
  const float room = fminf(8.f / c, 1e30f);
  const int last = (q0 + kRows < s.len ? q0 + kRows : s.len) - 1;   // last row of this tile
  const int steps = last / kStep + 1;
  for (int t = 0; t < steps; ++t) {
    DR_WAIT_VM(0);
    DR_LDS_SYNC();
    if (t + 1 < steps) load(t + 1);
    const int k0 = t * kStep;
    if (k0 > qw + 31) continue;   // all of this wave's rows come before these keys
    const TilePlace<D> tp = place.begin((t & 1) * (2 * kTile));
    f32x16 p[2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) p[x][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x) p[x] = mma32(read_rows<D>(lds, tp, 0, 32 * x, ks), qf[ks], p[x]);
    // four reads ahead of the products (as compiled otherwise two: 4 % slower on
    // sequences of 4096)
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    if (k0 == qw) {   // the wave's own rows are the step's first half, or its second
      mask_diagonal<true>(p[0], -INFINITY);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[1][r] = -INFINITY;
    } else if (k0 + 32 == qw) {
      mask_diagonal<true>(p[1], -INFINITY);
    }
    float top = p[0][0];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, p[x][r]);
    if (__any(top > m + room)) {
      top = fmaxf(m, max_halves(top));
      const float alpha = __builtin_amdgcn_exp2f((m - top) * c);
      m = top;
      sum *= alpha;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) o[cb] *= alpha;
    }
    const float mc = m * c;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[x][r] = __builtin_amdgcn_exp2f(p[x][r] * c - mc);
        sum += p[x][r];
      }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const u32x4 pf = c_operand(p[x], ks);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) o[cb] = mma32(read_cols<D>(lds, tp, kTile, 32 * x + 16 * ks, cb), pf, o[cb]);
      }
  }
  sum = sum_halves(sum);
  static_assert(kWaves * store_bytes<D> <= 4 * kTile, "rows of o in LDS");
  DR_LDS_SYNC();
  store_rows<D>(lds + w * store_bytes<D>, a.o + (s.first + qw) * a.ldo + hb, a.ldo, s.len - qw, o, 1.0f / sum, lane);
  if (row < s.len && h == 0) a.lse[(long long)head * a.b.rows + s.first + row] = m * a.scale + __logf(sum);
}

// Few tiles: 32 rows a workgroup, whose four waves take the steps of keys in turn, each
// with stages of its own (no barrier in the loop), and are joined at the end: four times
// the workgroups, each a quarter as long, for four times the reads of K and V.
template <int D>
__global__ __launch_bounds__(kThreads, 1) void attn_few_kernel(FwdArgs a) {
  constexpr int kKeys = 4096 / D;               // of a step: 16 KB of K and V
  constexpr int kTile = kKeys * D * 2, kMine = 4 * kTile, kBlocks = kKeys / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kWaves * kMine];   // two stages of K, V a wave
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place at;
  if (!place_of(a.grid, a.b, at)) return;
  const int tile = at.place, head = at.khead * (int)a.grid.per.d + at.g;
  const Seq s = sequence(a.b, at.seq);
  const int q0 = tile * kFewRows;
  const unsigned hb = (unsigned)head * (D * 2), kb = (unsigned)at.khead * (D * 2);
  zero_padding<D, kFewRows>(a, s, q0, tile == at.tiles - 1, head, hb);
  if (q0 >= s.len) return;

  const unsigned char* kp = a.k + s.first * a.ldk + kb;
  const unsigned char* vp = a.v + s.first * a.ldv + kb;
  const unsigned ldk = (unsigned)a.ldk, ldv = (unsigned)a.ldv;
  TileLoad<D, kKeys, 1> lk, lv;
  lk.init(0, lane, ldk);
  lv.init(0, lane, ldv);
  const unsigned lds0 = lds_offset(lds) + w * kMine;
  auto load = [&](int t, int stage) {   // (past the last row: zeros)
    const unsigned st = lds0 + stage * (2 * kTile);
    lk.issue(kp + (long long)t * kKeys * ldk, s.len - t * kKeys, ldk, st, 0);
    lv.issue(vp + (long long)t * kKeys * ldv, s.len - t * kKeys, ldv, st + kTile, 0);
  };
  const int row = q0 + (lane & 31);
  u32x4 qf[D / 16];
  row_fragments<D>(a.q + (s.first + row) * a.ldq + hb, row < s.len, lane, qf);
#pragma unroll
  for (int x = 0; x < D / 16; ++x) arrived(qf[x]);
  TilePlace<D> place;
  place.init(lane);
  place.rows += w * kMine, place.cols += w * kMine;
  f32x16 o[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[cb][r] = 0.f;
  float m = -INFINITY, sum = 0.f;
  const float c = a.scale * kLog2e, room = fminf(8.f / c, 1e30f);
  const int steps = (q0 + kFewRows - 1) / kKeys + 1;
  constexpr int kLoads = 2 * TileLoad<D, kKeys, 1>::kCount;   // of a step
  if (w < steps) load(w, 0);
  for (int t = w, st = 0; t < steps; t += kWaves, st ^= 1) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the other stage's reads are done)
    load(t + kWaves, st ^ 1);
    DR_WAIT_VM(kLoads);
    const int k0 = t * kKeys;
    const TilePlace<D> tp = place.begin(st * (2 * kTile));
    f32x16 p[kBlocks];
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) p[x][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int x = 0; x < kBlocks; ++x) p[x] = mma32(read_rows<D>(lds, tp, 0, 32 * x, ks), qf[ks], p[x]);
    if (t == steps - 1) {   // the rows' own block, and one after them
      if (kBlocks == 1 || k0 + 32 == q0) {
        mask_diagonal<true>(p[kBlocks - 1], -INFINITY);
      } else {
        mask_diagonal<true>(p[0], -INFINITY);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[kBlocks - 1][r] = -INFINITY;
      }
    }
    float top = p[0][0];
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, p[x][r]);
    if (__any(top > m + room)) {
      top = fmaxf(m, max_halves(top));
      const float alpha = __builtin_amdgcn_exp2f((m - top) * c);
      m = top;
      sum *= alpha;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) o[cb] *= alpha;
    }
    const float mc = m * c;
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[x][r] = __builtin_amdgcn_exp2f(p[x][r] * c - mc);
        sum += p[x][r];
      }
#pragma unroll
    for (int x = 0; x < kBlocks; ++x)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const u32x4 pf = c_operand(p[x], ks);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) o[cb] = mma32(read_cols<D>(lds, tp, kTile, 32 * x + 16 * ks, cb), pf, o[cb]);
      }
  }
  sum = sum_halves(sum);
  DR_WAIT_VM(0);
  DR_LDS_SYNC();
  // the waves' statistics, then their sums of O relative to the common maximum
  float* stat = reinterpret_cast<float*>(lds);   // [waves][m, sum][32]
  if (h == 0) stat[w * 64 + lane] = m, stat[w * 64 + 32 + lane] = sum;
  __syncthreads();
  float top = stat[lane & 31], total = 0.f;
#pragma unroll
  for (int i = 1; i < kWaves; ++i) top = fmaxf(top, stat[i * 64 + (lane & 31)]);
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    // (a wave without a step has m = -inf and sum 0; one whose scores are all NaN has sum NaN)
    const float mi = stat[i * 64 + (lane & 31)], scale = mi == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mi - top) * c);
    total = fmaf(stat[i * 64 + 32 + (lane & 31)], scale, total);
  }
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c) / total;
  if (w == 0 && h == 0 && row < s.len) a.lse[(long long)head * a.b.rows + s.first + row] = top * a.scale + __logf(total);
  join_waves<D>(lds + 1024, o, f, a.o + (s.first + q0) * a.ldo + hb, a.ldo, s.len - q0, w, lane);
}

}  // namespace
}  // namespace attn
}  // namespace dr

extern "C" dr_status dr_attention(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                  int64_t rows, int64_t N, int64_t T, const int32_t* off, const int32_t* len, int Hq, int Hkv,
                                  int64_t D, dr_dtype dtype, float scale, void* o, int64_t ldo, float* lse, void* stream) {
  using namespace dr;
  using namespace dr::attn;
  const dr_status st = check_batch(rows, N, T, off, Hq, Hkv, D, dtype, scale);
  if (st != DR_OK) return st;
  if (!good_rows(q, ldq, Hq, D, rows) || !good_rows(k, ldk, Hkv, D, rows) || !good_rows(v, ldv, Hkv, D, rows) ||
      !good_rows(o, ldo, Hq, D, rows) || (rows > 0 && !lse))
    return DR_ERR_ARG;
  if (rows == 0) return DR_OK;
  FwdArgs a = {};
  a.q = (const unsigned char*)q;
  a.k = (const unsigned char*)k;
  a.v = (const unsigned char*)v;
  a.o = (unsigned char*)o;
  a.lse = lse;
  a.ldq = ldq * 2, a.ldk = ldk * 2, a.ldv = ldv * 2, a.ldo = ldo * 2;
  a.b = Batch{off, len, rows, T, (int)N};
  a.Hq = Hq;
  a.scale = scale;
  dim3 grid;
  const bool few = few_tiles(a.b, Hq);
  if (!grid_of(a.b, few ? kFewRows : kRows, Hkv, Hq / Hkv, a.grid, grid)) return DR_ERR_UNSUPPORTED;
  if (few && D == 64) attn_few_kernel<64><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  else if (few) attn_few_kernel<128><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  else if (D == 64) attn_kernel<64><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  else attn_kernel<128><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  return launch_status();
}

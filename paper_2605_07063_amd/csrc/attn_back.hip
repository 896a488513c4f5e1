// Gradient of causal attention (dr_attention_backward).
//
//   P = exp(scale Q K^T - lse),  delta = rowsum(dO o O),
//   dS = P o (dO V^T - delta),   dQ = scale dS K,
//   dV = P^T dO,                 dK = scale dS^T Q,  summed over the query
//   heads that share a key head.
//
// Two kernels, so that every sum has one owner and a fixed order (no atomics):
// one over query tiles (dQ, and delta on the way), one over key tiles (dK, dV).
// Both recompute P, which costs seven products of the tile instead of five.  In
// each, a lane of a wave holds one of the wave's 32 own rows, and what it
// recomputes is the B operand of the product that follows without leaving its
// lanes (see attn.h).  P and dS are rounded to bf16 for those products; all
// sums are fp32.
//
// Bound by the MFMA and the VALU work around it, which wait for each other in the
// two waves of a SIMD that the registers allow (222 and 252 of 256 with D = 128).
// Full sequences of 4096, 32 query heads of 8 key heads, D = 128, four of them: dq
// 0.81 ms and dkv 1.11 (1.02 and 0.99 PFLOP/s; MFMA busy 0.57 and 0.55 at the 1.6 and
// 1.7 GHz that power leaves), 16 of 1024: 0.32 and 0.35 ms, MFMA busy 0.38 and 0.48.
// D = 64: 72 examples of 128 to 512 tokens 0.15 and 0.13 ms.  Slower: keys in pairs of
// waves that share P through LDS (1.60 ms instead of 1.18), 64 keys a wave (spills
// with D = 128; 1.09 ms and 0.93 with D = 64), eight waves a workgroup.
#include "attn.h"

namespace dr {
namespace attn {
namespace {

constexpr int kStep = 64;   // rows of a streamed tile

struct BackArgs {
  const unsigned char *q, *k, *v, *o, *g;   // g: gradient of o
  unsigned char *dq, *dk, *dv;
  const float* lse;                         // [Hq][rows]
  float *delta, *lse2;                      // [Hq][rows]: rowsum(dO o O), lse in powers of two
  long long ldq, ldk, ldv, ldo, ldg, lddq, lddk, lddv;
  Batch b;
  Grid grid;
  int Hq, Hkv, G;          // G: query heads per key head
  int parts;               // split dK, dV: parts of those, and their sums
  unsigned char *pk, *pv;  // fp32 [parts][rows][Hkv][D]
  float scale;
};

// padding of the slot in a tile of OWN rows from q0 on
template <int D, int OWN>
__device__ __forceinline__ void zero_dq(const BackArgs& a, const Seq& s, int q0, bool last, unsigned hb) {
  const long long from = q0 < s.len ? (s.len < q0 + OWN ? s.len : q0 + OWN) : q0;
  long long to = s.end - s.first;
  if (!last && q0 + OWN < to) to = q0 + OWN;
  if (from < to) zero_rows<D * 2>(a.dq + s.first * a.lddq + hb, a.lddq, from, to);
}
// rowsum(dO o O) of this lane's row
template <int D>
__device__ __forceinline__ float row_delta(const u32x4 (&of)[D / 16], const u32x4 (&gf)[D / 16]) {
  float delta = 0.f;
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      delta = fmaf(__uint_as_float(of[x][e] << 16), __uint_as_float(gf[x][e] << 16), delta);
      delta = fmaf(__uint_as_float(of[x][e] & 0xffff0000u), __uint_as_float(gf[x][e] & 0xffff0000u), delta);
    }
  return sum_halves(delta);
}
// P^T and dP^T of the 32 keys at row0 of a stage; keys after a row get zeros in both
template <int D>
__device__ __forceinline__ void dq_block(const unsigned char* lds, const TilePlace<D>& tp, int tile, int row0, bool diag,
                                         const u32x4 (&qf)[D / 16], const u32x4 (&gf)[D / 16], float c, float lse2, f32x16& p,
                                         f32x16& dp) {
#pragma unroll
  for (int r = 0; r < 16; ++r) p[r] = 0.f, dp[r] = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    p = mma32(read_rows<D>(lds, tp, 0, row0, ks), qf[ks], p);
    dp = mma32(read_rows<D>(lds, tp, tile, row0, ks), gf[ks], dp);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(p[r] * c - lse2);
  if (diag) {
    asm volatile("");   // (a branch: without it the selections are made in every step)
    mask_diagonal<true>(p, 0.f);
    mask_diagonal<true>(dp, 0.f);
  }
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_dq_kernel(BackArgs a) {
  constexpr int kTile = kStep * D * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTile];   // two stages of K, V
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place at;
  if (!place_of(a.grid, a.b, at)) return;
  const int tile = at.place, head = at.khead * a.G + at.g;
  const Seq s = sequence(a.b, at.seq);
  const int q0 = tile * kRows;
  const unsigned hb = (unsigned)head * (D * 2), kb = (unsigned)at.khead * (D * 2);
  zero_dq<D, kRows>(a, s, q0, tile == at.tiles - 1, hb);
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
  load(0);
  TilePlace<D> place;
  place.init(lane);

  const int qw = q0 + 32 * w, row = qw + (lane & 31);
  const bool live = row < s.len;
  const long long stat = (long long)head * a.b.rows + s.first + row;
  u32x4 qf[D / 16], gf[D / 16];
  row_fragments<D>(a.q + (s.first + row) * a.ldq + hb, live, lane, qf);
  row_fragments<D>(a.g + (s.first + row) * a.ldg + hb, live, lane, gf);
  float delta;
  {
    u32x4 of[D / 16];
    row_fragments<D>(a.o + (s.first + row) * a.ldo + hb, live, lane, of);
    delta = row_delta<D>(of, gf);
  }
  float lse2 = live ? a.lse[stat] * kLog2e : 0.f;
  arrived(lse2);
#pragma unroll
  for (int x = 0; x < D / 16; ++x) arrived(qf[x]), arrived(gf[x]);

  f32x16 dq[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[cb][r] = 0.f;
  const float c = a.scale * kLog2e;
  const int last = (q0 + kRows < s.len ? q0 + kRows : s.len) - 1;
  const int steps = last / kStep + 1;
  auto block = [&](const TilePlace<D>& tp, int x, bool diag, f32x16& p, f32x16& dp) __attribute__((always_inline)) {
    dq_block<D>(lds, tp, kTile, 32 * x, diag, qf, gf, c, lse2, p, dp);
  };
  // delta is also sum_j P_j dP_j, and o is rounded to bf16: over the first rows of a
  // sequence, where few probabilities share it, that rounding weighs as much as the
  // one of dS.  For rows whose keys are all in the first step the sum is taken first;
  // the others leave dkv the exact delta, which is theirs plus the sum of dS.  (Errors
  // of dq and dk against fp64 on 72 sequences of 128 to 512 tokens: 2.6e-3 -> 2.5e-3,
  // on 61 of 1 to 2039 2.6e-3 -> 2.4e-3, where bf16 outputs alone have 1.7e-3; 0 to 4 %
  // of the backward's time.)
  float sum = 0.f;
  for (int t = 0; t < steps; ++t) {
    DR_WAIT_VM(0);
    DR_LDS_SYNC();
    if (t + 1 < steps) load(t + 1);
    const int k0 = t * kStep;
    const TilePlace<D> tp = place.begin((t & 1) * (2 * kTile));
    if (qw < kStep && t == 0) {
      delta = 0.f;
#pragma unroll 1
      for (int x = 0; 32 * x <= qw; ++x) {
        f32x16 p, dp;
        block(tp, x, 32 * x == qw, p, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) delta = fmaf(p[r], dp[r], delta);
      }
      delta = sum_halves(delta);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (k0 + 32 * x > qw) continue;   // these keys come after all of this wave's rows
      f32x16 p, dp;
      block(tp, x, k0 + 32 * x == qw, p, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] *= dp[r] - delta;
        sum += p[r];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const u32x4 pf = c_operand(p, ks);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) dq[cb] = mma32(read_cols<D>(lds, tp, 0, 32 * x + 16 * ks, cb), pf, dq[cb]);
      }
    }
  }
  sum = sum_halves(sum);
  if (live && h == 0) {
    a.delta[stat] = delta + sum;
    a.lse2[stat] = lse2;
  }
  static_assert(kWaves * store_bytes<D> <= 4 * kTile, "rows of dq in LDS");
  DR_LDS_SYNC();
  store_rows<D>(lds + w * store_bytes<D>, a.dq + (s.first + qw) * a.lddq + hb, a.lddq, s.len - qw, dq, a.scale, lane);
}

// Few tiles (see attn_few_kernel): 32 rows a workgroup, its waves take the steps in turn.
// (One sequence of 3488 tokens, 3 heads of 128: the whole backward 145 us with 128 rows
// and 100.)  The first 64 rows of a sequence, whose delta is summed from P and dP first,
// stay with one wave.
template <int D>
__global__ __launch_bounds__(kThreads, 1) void attn_dq_few_kernel(BackArgs a) {
  constexpr int kKeys = 4096 / D, kTile = kKeys * D * 2, kMine = 4 * kTile, kBlocks = kKeys / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kWaves * kMine];   // two stages of K, V a wave
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place at;
  if (!place_of(a.grid, a.b, at)) return;
  const int tile = at.place, head = at.khead * a.G + at.g;
  const Seq s = sequence(a.b, at.seq);
  const int q0 = tile * kFewRows;
  const unsigned hb = (unsigned)head * (D * 2), kb = (unsigned)at.khead * (D * 2);
  zero_dq<D, kFewRows>(a, s, q0, tile == at.tiles - 1, hb);
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
  const bool live = row < s.len;
  const long long stat = (long long)head * a.b.rows + s.first + row;
  u32x4 qf[D / 16], gf[D / 16];
  row_fragments<D>(a.q + (s.first + row) * a.ldq + hb, live, lane, qf);
  row_fragments<D>(a.g + (s.first + row) * a.ldg + hb, live, lane, gf);
  float delta;
  {
    u32x4 of[D / 16];
    row_fragments<D>(a.o + (s.first + row) * a.ldo + hb, live, lane, of);
    delta = row_delta<D>(of, gf);
  }
  float lse2 = live ? a.lse[stat] * kLog2e : 0.f;
  arrived(lse2);
#pragma unroll
  for (int x = 0; x < D / 16; ++x) arrived(qf[x]), arrived(gf[x]);
  TilePlace<D> place;
  place.init(lane);
  place.rows += w * kMine, place.cols += w * kMine;
  f32x16 dq[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[cb][r] = 0.f;
  const float c = a.scale * kLog2e;
  const bool alone = q0 < kStep;
  const int steps = alone && w > 0 ? 0 : (q0 + kFewRows - 1) / kKeys + 1, by = alone ? 1 : kWaves;
  constexpr int kLoads = 2 * TileLoad<D, kKeys, 1>::kCount;   // of a step
  float sum = 0.f;
  if (w < steps) load(w, 0);
  if (alone && w == 0) {
    if (steps > 1) load(1, 1);
    DR_WAIT_VM(0);
    delta = 0.f;
#pragma unroll 1
    for (int x = 0; 32 * x <= q0; ++x) {
      const TilePlace<D> tp = place.begin(kBlocks == 1 ? x * (2 * kTile) : x * (64 * D));
      f32x16 p, dp;
      dq_block<D>(lds, tp, kTile, 0, 32 * x == q0, qf, gf, c, lse2, p, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) delta = fmaf(p[r], dp[r], delta);
    }
    delta = sum_halves(delta);
  }
  for (int t = w, st = 0; t < steps; t += by, st ^= 1) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the other stage's reads are done)
    load(t + by, st ^ 1);
    DR_WAIT_VM(kLoads);
    const TilePlace<D> tp = place.begin(st * (2 * kTile));
#pragma unroll
    for (int x = 0; x < kBlocks; ++x) {
      const int k0 = t * kKeys + 32 * x;
      if (k0 > q0) continue;   // these keys come after all of the rows
      f32x16 p, dp;
      dq_block<D>(lds, tp, kTile, 32 * x, k0 == q0, qf, gf, c, lse2, p, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] *= dp[r] - delta;
        sum += p[r];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const u32x4 pf = c_operand(p, ks);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) dq[cb] = mma32(read_cols<D>(lds, tp, 0, 32 * x + 16 * ks, cb), pf, dq[cb]);
      }
    }
  }
  sum = sum_halves(sum);
  DR_WAIT_VM(0);
  DR_LDS_SYNC();
  float* sums = reinterpret_cast<float*>(lds);   // [waves][32]
  if (h == 0) sums[w * 32 + lane] = sum;
  __syncthreads();
  if (w == 0 && h == 0 && live) {
#pragma unroll
    for (int i = 0; i < kWaves; ++i) delta += sums[i * 32 + lane];
    a.delta[stat] = delta;
    a.lse2[stat] = lse2;
  }
  join_waves<D>(lds + 1024, dq, a.scale, a.dq + (s.first + q0) * a.lddq + hb, a.lddq, s.len - q0, w, lane);
}

// Own rows: 128 keys of one key head, 32 a wave; Q and dO of the query heads that
// share it stream through LDS, 64 rows a step, with their lse and delta.  Rows past
// the sequence's end arrive as zeros: their P is 1 but dO = 0.  With SPLIT a tile's
// steps are dealt to `parts` workgroups, whose sums go to the workspace and are joined
// by attn_join_kernel.
template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void attn_dkv_kernel(BackArgs a) {
  constexpr int kTile = kStep * D * 2, kStage = 2 * kTile + 2 * kStep * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place at;
  if (!place_of(a.grid, a.b, at)) return;
  const int head = at.khead;
  const Seq s = sequence(a.b, at.seq);
  // places count from the last tile that holds tokens, whose work is the least
  const int own = (s.len + kRows - 1) / kRows;
  const int tile = at.place < own ? own - 1 - at.place : at.place;
  const int n0 = tile * kRows;
  const unsigned kb = (unsigned)head * (D * 2);
  const long long part_ld = (long long)a.Hkv * (D * 4), part = (long long)at.g * a.b.rows * part_ld;
  {
    const long long from = n0 < s.len ? (s.len < n0 + kRows ? s.len : n0 + kRows) : n0;
    long long to = s.end - s.first;
    if (tile < at.tiles - 1 && n0 + kRows < to) to = n0 + kRows;
    if (from < to) {
      if constexpr (SPLIT) {
        zero_rows<D * 4>(a.pk + part + s.first * part_ld + 2 * kb, part_ld, from, to);
        zero_rows<D * 4>(a.pv + part + s.first * part_ld + 2 * kb, part_ld, from, to);
      } else {
        zero_rows<D * 2>(a.dk + s.first * a.lddk + kb, a.lddk, from, to);
        zero_rows<D * 2>(a.dv + s.first * a.lddv + kb, a.lddv, from, to);
      }
    }
  }
  if (n0 >= s.len) return;

  const unsigned ldq = (unsigned)a.ldq, ldg = (unsigned)a.ldg;
  TileLoad<D, kStep> lq, lg;
  lq.init(w, lane, ldq);
  lg.init(w, lane, ldg);
  const unsigned lds0 = lds_offset(lds);
  const int first = n0 / kStep, per = (s.len - 1) / kStep + 1 - first;   // query steps of one head
  const long long all = (long long)per * a.G;
  const int t0 = SPLIT ? (int)(at.g * all / a.parts) : 0, steps = (SPLIT ? (int)((at.g + 1) * all / a.parts) : (int)all) - t0;
  int lh = SPLIT ? t0 / per : 0, ls = first + t0 - lh * per;   // the step to load next
  int ms = ls;
  lh += head * a.G;
  auto load = [&](int t) {
    const unsigned st = lds0 + (t & 1) * kStage;
    const long long r0 = s.first + (long long)ls * kStep;
    const int n = s.len - ls * kStep;
    lq.issue(a.q + r0 * ldq + (long long)lh * (D * 2), n, ldq, st, w);
    lg.issue(a.g + r0 * ldg + (long long)lh * (D * 2), n, ldg, st + kTile, w);
    if (w < 2) {   // 64 values of lse (wave 0), of delta (wave 1): one dword a lane, zeros past the end
      const float* src = (w == 0 ? a.lse2 : a.delta) + (long long)lh * a.b.rows + r0;
      const unsigned long long b = reinterpret_cast<unsigned long long>(src);
      const u32x4 rsrc = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)b),
                          (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(b >> 32)) & 0xffffu,
                          (unsigned)__builtin_amdgcn_readfirstlane(4 * (n < kStep ? n : kStep)), 0x00020000u};
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds"
                   :: "s"(st + 2 * kTile + w * (kStep * 4)), "v"(lane * 4), "s"(rsrc) : "memory", "m0");
    }
    if (++ls == first + per) {
      ls = first;
      ++lh;
    }
  };
  if (!SPLIT || steps > 0) load(0);
  TilePlace<D> place;
  place.init(lane);

  const int nw = n0 + 32 * w, row = nw + (lane & 31);   // this wave's first key, this lane's
  const bool live = row < s.len;
  u32x4 kf[D / 16], vf[D / 16];
  row_fragments<D>(a.k + (s.first + row) * a.ldk + kb, live, lane, kf);
  row_fragments<D>(a.v + (s.first + row) * a.ldv + kb, live, lane, vf);
#pragma unroll
  for (int x = 0; x < D / 16; ++x) arrived(kf[x]), arrived(vf[x]);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[cb][r] = 0.f, dv[cb][r] = 0.f;
  const float c = a.scale * kLog2e;
  for (int t = 0; t < steps; ++t) {
    DR_WAIT_VM(0);
    DR_LDS_SYNC();
    if (t + 1 < steps) load(t + 1);
    const int step0 = ms * kStep;
    if (++ms == first + per) ms = first;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int x0 = 32 * x, m0 = step0 + x0;   // this wave's first query row
      if (m0 < nw) continue;   // they come before all of this wave's keys
      const TilePlace<D> tp = place.begin((t & 1) * kStage + x0 * (2 * D));
      const float* st = reinterpret_cast<const float*>(lds + (t & 1) * kStage + 2 * kTile) + x0;
      f32x16 p, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = 0.f, dp[r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        p = mma32(read_rows<D>(lds, tp, 0, 0, ks), kf[ks], p);
        dp = mma32(read_rows<D>(lds, tp, kTile, 0, ks), vf[ks], dp);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(st + 8 * q + 4 * h);
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(st + kStep + 8 * q + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * q + e;
          p[r] = __builtin_amdgcn_exp2f(p[r] * c - l4[e]);
          dp[r] = p[r] * (dp[r] - d4[e]);
        }
      }
      if (m0 == nw) {
        asm volatile("");   // (a branch: without it the selections are made in every step)
        mask_diagonal<false>(p, 0.f);
        mask_diagonal<false>(dp, 0.f);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const u32x4 pf = c_operand(p, ks), df = c_operand(dp, ks);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) {
          dv[cb] = mma32(read_cols<D>(lds, tp, kTile, 16 * ks, cb), pf, dv[cb]);
          dk[cb] = mma32(read_cols<D>(lds, tp, 0, 16 * ks, cb), df, dk[cb]);
        }
      }
    }
  }
  if constexpr (SPLIT) {
    if (!live) return;
    unsigned char* ok = a.pk + part + (s.first + row) * part_ld + 2 * kb + 16 * h;
    unsigned char* ov = a.pv + part + (s.first + row) * part_ld + 2 * kb + 16 * h;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      *reinterpret_cast<f32x4*>(ok + 32 * i) =
          f32x4{dk[i / 4][4 * (i % 4)], dk[i / 4][4 * (i % 4) + 1], dk[i / 4][4 * (i % 4) + 2], dk[i / 4][4 * (i % 4) + 3]};
      *reinterpret_cast<f32x4*>(ov + 32 * i) =
          f32x4{dv[i / 4][4 * (i % 4)], dv[i / 4][4 * (i % 4) + 1], dv[i / 4][4 * (i % 4) + 2], dv[i / 4][4 * (i % 4) + 3]};
    }
  } else {
    static_assert(kWaves * store_bytes<D> <= 2 * kStage, "rows of dk, dv in LDS");
    DR_LDS_SYNC();
    unsigned char* mine = lds + w * store_bytes<D>;
    // (the lane's number once more: no register holds it over the loop)
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    store_rows<D>(mine, a.dk + (s.first + nw) * a.lddk + kb, a.lddk, s.len - nw, dk, a.scale, l);
    store_rows<D>(mine, a.dv + (s.first + nw) * a.lddv + kb, a.lddv, s.len - nw, dv, 1.f, l);
  }
}

// dk, dv from the parts' sums, in order: four values a thread
__global__ __launch_bounds__(kThreads) void attn_join_kernel(BackArgs a, int D) {
  const long long n = a.b.rows * a.Hkv * D, i = ((long long)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (i >= n) return;
  f32x4 k = {0.f, 0.f, 0.f, 0.f}, v = k;
  for (int p = 0; p < a.parts; ++p) {
    k += *reinterpret_cast<const f32x4*>(a.pk + (p * n + i) * 4);
    v += *reinterpret_cast<const f32x4*>(a.pv + (p * n + i) * 4);
  }
  k *= a.scale;
  const long long row = i / ((long long)a.Hkv * D), col = i % ((long long)a.Hkv * D);
  *reinterpret_cast<uint2*>(a.dk + row * a.lddk + 2 * col) = uint2{pack2(k[0], k[1]), pack2(k[2], k[3])};
  *reinterpret_cast<uint2*>(a.dv + row * a.lddv + 2 * col) = uint2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}

}  // namespace
}  // namespace attn
}  // namespace dr

namespace dr {
namespace attn {
namespace {

// Parts that a tile's steps (64 query rows of one head) are dealt to for dK and dV: as
// many as bring the workgroups past 640, at most 8 and with 4 steps in each of the
// longest tile's.  The sums of the parts cost 16 bytes written and read per value of
// dK and dV and part.  The whole backward: with 1024 workgroups (16 x 1024 rows of 8
// key heads, D = 128) two parts take 0.64 ms and one 0.55; with 256 (one sequence of
// 4096) three take 0.52 ms and one 0.86, with 84 (one of 3488, 3 heads) eight 0.15 and
// one 0.23, with 64 (two of 4096, one key head, D = 64) eight 0.20 and one 0.72.
// (Parts for the longest tiles alone: 0.61 ms with 256; fewer and more equal
// workgroups leave CUs idle at the end.)  None where the longest workgroup's steps are
// few beside the number of workgroups, whose sums would cost more than that saves: 64
// examples of 331 tokens (384 workgroups of at most 18 steps; 6 / 2 heads of 128) 109
// us whole and 145 in three parts, 12 of 477 (192 of 24; 12 / 4 heads) 105 and 90.  Over
// 240 shapes of 60 to 576 workgroups of 2 to 256 steps (D = 64, 128; 1 to 8 query heads a
// key head; 100 to 2000 tokens) the parts' time over the whole's is 1.10 to 1.72 where 9
// steps are 0.13 to 0.5 of the workgroups and there are steps to deal, 0.91 to 1.10 between
// 0.8 and 1.25, 0.65 to 0.99 from 1.4 to 4, and down to 0.26 above.
int most_parts(int64_t groups) {
  const int64_t p = (639 + groups) / groups;
  return (int)(p < 8 ? p : 8);
}
int parts_of(const Batch& b, int Hkv, int G) {
  const int64_t tiles = (b.T + kRows - 1) / kRows, packed = (b.rows + kRows - 1) / kRows;
  const int64_t groups = (b.off ? (packed > b.N ? packed : b.N) : b.N * (tiles > 1 ? tiles : 1)) * Hkv;
  const int64_t steps = 2 * tiles * G, p = most_parts(groups), most = steps / 4;
  return 9 * steps <= groups || most < 1 ? 1 : (int)(p < most ? p : most);
}
// delta, lse2, then the parts' sums
size_t stat_bytes(int64_t rows, int Hq) { return align_up((size_t)rows * (size_t)Hq * sizeof(float), 256); }
size_t part_bytes(int64_t rows, int Hq, int Hkv, int64_t D) {
  const int parts = most_parts((rows + kRows - 1) / kRows * Hkv);
  return parts > 1 ? (size_t)parts * (size_t)rows * (size_t)Hkv * (size_t)D * sizeof(float) : 0;
}

template <int D>
void launch_back(const BackArgs& a, const Grid& gq, dim3 nq, const Grid& gk, dim3 nk, bool few, hipStream_t hs) {
  BackArgs b = a;
  b.grid = gq;
  if (few) attn_dq_few_kernel<D><<<nq, kThreads, 0, hs>>>(b);
  else attn_dq_kernel<D><<<nq, kThreads, 0, hs>>>(b);
  b.grid = gk;
  if (a.parts == 1) {
    attn_dkv_kernel<D, false><<<nk, kThreads, 0, hs>>>(b);
    return;
  }
  attn_dkv_kernel<D, true><<<nk, kThreads, 0, hs>>>(b);
  const int64_t n = a.b.rows * a.Hkv * D / 4;
  attn_join_kernel<<<(int)((n + kThreads - 1) / kThreads), kThreads, 0, hs>>>(b, D);
}

}  // namespace
}  // namespace attn
}  // namespace dr

extern "C" size_t dr_attention_workspace_size(int64_t rows, int Hq, int Hkv, int64_t D) {
  using namespace dr::attn;
  if (rows < 1 || Hq < 1 || Hkv < 1 || D < 1 || Hq % Hkv) return 0;
  return 2 * stat_bytes(rows, Hq) + 2 * part_bytes(rows, Hq, Hkv, D);
}

extern "C" dr_status dr_attention_backward(const void* g, int64_t ldg, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                           const void* v, int64_t ldv, const void* o, int64_t ldo, const float* lse,
                                           int64_t rows, int64_t N, int64_t T, const int32_t* off, const int32_t* len, int Hq,
                                           int Hkv, int64_t D, dr_dtype dtype, float scale, void* dq, int64_t lddq, void* dk,
                                           int64_t lddk, void* dv, int64_t lddv, void* workspace, size_t ws_bytes,
                                           void* stream) {
  using namespace dr;
  using namespace dr::attn;
  const dr_status st = check_batch(rows, N, T, off, Hq, Hkv, D, dtype, scale);
  if (st != DR_OK) return st;
  if (!good_rows(g, ldg, Hq, D, rows) || !good_rows(q, ldq, Hq, D, rows) || !good_rows(k, ldk, Hkv, D, rows) ||
      !good_rows(v, ldv, Hkv, D, rows) || !good_rows(o, ldo, Hq, D, rows) || !good_rows(dq, lddq, Hq, D, rows) ||
      !good_rows(dk, lddk, Hkv, D, rows) || !good_rows(dv, lddv, Hkv, D, rows) || (rows > 0 && !lse))
    return DR_ERR_ARG;
  if (rows == 0) return DR_OK;
  if (workspace && !aligned16(workspace)) return DR_ERR_ARG;
  if (!workspace || ws_bytes < dr_attention_workspace_size(rows, Hq, Hkv, D)) return DR_ERR_WORKSPACE;
  BackArgs a = {};
  a.q = (const unsigned char*)q;
  a.k = (const unsigned char*)k;
  a.v = (const unsigned char*)v;
  a.o = (const unsigned char*)o;
  a.g = (const unsigned char*)g;
  a.dq = (unsigned char*)dq;
  a.dk = (unsigned char*)dk;
  a.dv = (unsigned char*)dv;
  a.lse = lse;
  unsigned char* ws = (unsigned char*)workspace;
  a.delta = (float*)ws;
  a.lse2 = (float*)(ws + stat_bytes(rows, Hq));
  a.pk = ws + 2 * stat_bytes(rows, Hq);
  a.pv = a.pk + part_bytes(rows, Hq, Hkv, D);
  a.ldq = ldq * 2, a.ldk = ldk * 2, a.ldv = ldv * 2, a.ldo = ldo * 2, a.ldg = ldg * 2;
  a.lddq = lddq * 2, a.lddk = lddk * 2, a.lddv = lddv * 2;
  a.b = Batch{off, len, rows, T, (int)N};
  a.Hq = Hq, a.Hkv = Hkv, a.G = Hq / Hkv;
  a.parts = parts_of(a.b, Hkv, a.G);
  a.scale = scale;
  const hipStream_t hs = (hipStream_t)stream;
  Grid gq, gk;
  dim3 nq, nk;
  const bool few = few_tiles(a.b, Hq);
  if (!grid_of(a.b, few ? kFewRows : kRows, Hkv, a.G, gq, nq) || !grid_of(a.b, kRows, Hkv, a.parts, gk, nk) ||
      rows > (int64_t)0x7fffffff * 4 * kThreads / (Hkv * D))
    return DR_ERR_UNSUPPORTED;
  if (D == 64) launch_back<64>(a, gq, nq, gk, nk, few, hs);
  else launch_back<128>(a, gq, nq, gk, nk, few, hs);
  return launch_status();
}

// Per-head norm of queries and keys with the position rotation in the same
// pass (dr_qk_norm_rope), and its gradient (dr_qk_norm_rope_backward).
//
//   y = x * r * w,  r = (mean(x^2) + eps)^(-1/2) over the head's D values,
//   out = R(pos) y, R a rotation of D / 2 pairs by the table's angles;
//   dy = R^T dout,  dw = sum over rows and heads of dy * x * r,
//   dx = r * (w dy - x r^2 mean(w dy x)).
//
// Bound by HBM: every value of q and k is read once and written once (the
// backward reads two tensors and writes one), all arithmetic in fp32 registers,
// one rounding at the store.  A lane holds 16 bytes from each half of a head, so
// that with pairs (i, i + D/2) both members of a pair are its own, and with
// pairs (2i, 2i + 1) anyway; D / 2 * 16 bytes make 4 to 16 lanes a head, whose
// sums are DPP exchanges.  A wave takes the heads of one row, 64 / lanes at a
// time, with the row's angles in registers: the table (fp32, twice the bytes of
// one bf16 head) is read once per row and not once per head.  bf16, D = 128: 16384 rows
// of 40 heads out of the fused projection, rotated only, 64 us (5.2 TB/s, where a copy
// reaches 4.9); 36864 rows of 24 heads with norms 79 us, their gradients 134 us (680 MB).
// Of a batch with padding (72 slots of 512 of those rows, 128 to 512 tokens in each: 0.62 are
// tokens) 77 and 120 us in calls of their own, where all rows take 86 and 135: padding rows
// are written, not read.  The same tokens packed, with offsets, 57 and 87.
#include "attn.h"   // the batch's rows

namespace dr {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxBackBlocks = 768;    // partial sums of the norms' weight gradients: one round of what is
                                       // resident (1024 blocks: 7 % slower, in two rounds)
constexpr int kSumCols = 16;           // columns of them per block of the final sum,
constexpr int kSumThreads = 1024;      // and its threads

struct RopeArgs {
  const unsigned char *q, *k, *gq, *gk;   // gq, gk: gradients of the outputs (backward)
  unsigned char *oq, *ok;                 // outputs, or gradients of the inputs
  long long ldq, ldk, ldgq, ldgk, ldoq, ldok;   // bytes between rows
  long long rows, T, table_rows;
  const float *wq, *wk, *table;
  const int* pos;
  float eps;
  int Hq, H;        // query heads, all heads
  float* partial;   // backward: [blocks][2][D]
  bool batch;       // sequences with padding, or packed ones
  attn::Batch b;
  attn::Divisor perT;
};

template <bool BF16, int N>
__device__ __forceinline__ void load_vals(const unsigned char* p, float (&v)[N]) {
  const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
      v[i] = __uint_as_float(u[i]);
    }
  }
}
template <bool BF16, int N>
__device__ __forceinline__ void store_vals(unsigned char* p, const float (&v)[N]) {
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    else u[i] = __float_as_uint(v[i]);
  }
  *reinterpret_cast<u32x4*>(p) = u;
}

template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, false));
}
// sum over groups of L lanes (4, 8 or 16), the same in each of them
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp_f<0xB1>(v);                       // quad_perm [1, 0, 3, 2]
  v += dpp_f<0x4E>(v);                       // quad_perm [2, 3, 0, 1]
  if constexpr (L >= 8) v += dpp_f<0x141>(v);   // row_half_mirror
  if constexpr (L >= 16) v += dpp_f<0x140>(v);  // row_mirror
  return v;
}

// N values from each half of a head: chunk 0 = columns [N j, N j + N), chunk 1
// = the same D / 2 further on.  c, s hold the N angles of chunk 0's and chunk
// 1's pairs: with halves pair i is (chunk 0, chunk 1)[i]; with neighbours chunk
// 0 holds pairs 0 .. N/2 - 1 of the lane's angles and chunk 1 the others.
template <bool PAIRS, int N>
__device__ __forceinline__ void turn(float (&a)[N], float (&b)[N], const float (&c)[N], const float (&s)[N], float sgn) {
  if constexpr (PAIRS) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float a0 = a[2 * i], a1 = a[2 * i + 1], b0 = b[2 * i], b1 = b[2 * i + 1];
      const float s0 = sgn * s[i], s1 = sgn * s[N / 2 + i];
      a[2 * i] = a0 * c[i] - a1 * s0;
      a[2 * i + 1] = a0 * s0 + a1 * c[i];
      b[2 * i] = b0 * c[N / 2 + i] - b1 * s1;
      b[2 * i + 1] = b0 * s1 + b1 * c[N / 2 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = a[i], y = b[i], si = sgn * s[i];
      a[i] = x * c[i] - y * si;
      b[i] = x * si + y * c[i];
    }
  }
}

// The packed sequence whose slot holds the row (uniform): the last one that starts no later,
// found by the wave's lanes in steps of 64 to one.
__device__ __forceinline__ int sequence_of(const attn::Batch& b, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  for (int n = b.N; n > 1;) {
    const int step = (n + 63) / 64, at = lane * step;
    const int starts = __popcll(__ballot(at < n && b.off[lo + (at < n ? at : 0)] <= row));
    const int skip = starts > 1 ? (starts - 1) * step : 0;
    lo += skip;
    n = n - skip < step ? n - skip : step;
  }
  return lo;
}
// Whether the row is a token, and its position, clamped into the table: pos[row], or its
// place in its sequence.  BATCH: the row is uniform; the kernels without it keep theirs (with
// one kernel for both: rope_train 225 us, 223 without).
template <bool BATCH>
__device__ __forceinline__ bool token(const RopeArgs& a, long long row, long long& p) {
  long long at;
  bool is = true;
  if constexpr (BATCH) {
    const int seq = a.b.off ? sequence_of(a.b, (int)row) : (int)attn::over((unsigned)row, a.perT);
    const attn::Seq s = attn::sequence(a.b, seq);
    at = row - s.first;
    is = at >= 0 && at < s.len;
  } else {
    at = a.pos ? 0 : row % a.T;
  }
  p = a.pos ? (long long)a.pos[row] : at;
  p = p < 0 ? 0 : (p >= a.table_rows ? a.table_rows - 1 : p);
  return is;
}
// this wave's number: uniform where rows are looked up
template <bool BATCH>
__device__ __forceinline__ int wave() {
  const int w = threadIdx.x >> 6;
  return BATCH ? __builtin_amdgcn_readfirstlane(w) : w;
}
// zeros in the row's outputs
template <int ROW>   // bytes of a head
__device__ __forceinline__ void zero_row(const RopeArgs& a, long long row, int lane) {
  for (int i = lane; i < a.H * (ROW / 16); i += 64) {
    const int q = a.Hq * (ROW / 16);
    unsigned char* o = i < q ? a.oq + row * a.ldoq + i * 16ll : a.ok + row * a.ldok + (i - q) * 16ll;
    *reinterpret_cast<u32x4*>(o) = u32x4{0u, 0u, 0u, 0u};
  }
}

// the lane's N angles at position p
template <bool PAIRS, int N, int D>
__device__ __forceinline__ void load_angles(const RopeArgs& a, long long p, int j, float (&c)[N], float (&s)[N]) {
  const f32x4* t = reinterpret_cast<const f32x4*>(a.table + p * D);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {   // two (cos, sin) pairs each
    const int pair = PAIRS ? (i < N / 4 ? j * (N / 2) + 2 * i : D / 4 + j * (N / 2) + 2 * i - N / 2) : j * N + 2 * i;
    const f32x4 v = t[pair / 2];
    c[2 * i] = v[0];
    s[2 * i] = v[1];
    c[2 * i + 1] = v[2];
    s[2 * i + 1] = v[3];
  }
}

template <int N>
__device__ __forceinline__ void load_weight(const float* w, int col, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const f32x4 u = reinterpret_cast<const f32x4*>(w + col)[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * i + e] = u[e];
  }
}

template <bool BF16, int D, bool PAIRS, bool NORM, bool BATCH>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  constexpr int N = BF16 ? 8 : 4, L = D / 2 / N, E = BF16 ? 2 : 4, HPW = 64 / L;
  const int lane = threadIdx.x & 63, j = lane % L, hl = lane / L;
  const long long row = (long long)blockIdx.x * kWaves + wave<BATCH>();
  if (row >= a.rows) return;
  long long p;
  if (!token<BATCH>(a, row, p)) {
    zero_row<D * E>(a, row, lane);
    return;
  }
  float c[N], s[N];
  load_angles<PAIRS, N, D>(a, p, j, c, s);
  for (int h = hl; h < a.H; h += HPW) {
    const bool isq = h < a.Hq;
    const long long at = (long long)(isq ? h : h - a.Hq) * (D * E) + j * 16;
    const unsigned char* x = (isq ? a.q + row * a.ldq : a.k + row * a.ldk) + at;
    unsigned char* o = (isq ? a.oq + row * a.ldoq : a.ok + row * a.ldok) + at;
    float u[N], v[N];
    load_vals<BF16>(x, u);
    load_vals<BF16>(x + D / 2 * E, v);
    if constexpr (NORM) {
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) sq += u[i] * u[i] + v[i] * v[i];
      const float r = 1.0f / sqrtf(group_sum<L>(sq) * (1.0f / D) + a.eps);
      const float* w = isq ? a.wq : a.wk;
      float w0[N], w1[N];
      load_weight(w, j * N, w0);
      load_weight(w, j * N + D / 2, w1);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        u[i] = u[i] * r * w0[i];
        v[i] = v[i] * r * w1[i];
      }
    }
    turn<PAIRS>(u, v, c, s, 1.f);
    store_vals<BF16>(o, u);
    store_vals<BF16>(o + D / 2 * E, v);
  }
}

// A block takes rows in strides of the grid; a lane keeps its columns' sums of
// dy * x * r for queries and for keys, which the block joins in LDS in a fixed
// order and leaves as one partial row.
template <bool BF16, int D, bool PAIRS, bool NORM, bool BATCH>
__global__ __launch_bounds__(kThreads) void rope_back_kernel(RopeArgs a) {
  constexpr int N = BF16 ? 8 : 4, L = D / 2 / N, E = BF16 ? 2 : 4, HPW = 64 / L;
  const int lane = threadIdx.x & 63, j = lane % L, hl = lane / L;
  float sum[2][2 * N] = {};
  for (long long row = (long long)blockIdx.x * kWaves + wave<BATCH>(); row < a.rows;
       row += (long long)gridDim.x * kWaves) {
    long long p;
    if (!token<BATCH>(a, row, p)) {
      zero_row<D * E>(a, row, lane);
      continue;
    }
    float c[N], s[N];
    load_angles<PAIRS, N, D>(a, p, j, c, s);
    for (int h = hl; h < a.H; h += HPW) {
      const bool isq = h < a.Hq;
      const long long at = (long long)(isq ? h : h - a.Hq) * (D * E) + j * 16;
      const unsigned char* g = (isq ? a.gq + row * a.ldgq : a.gk + row * a.ldgk) + at;
      unsigned char* o = (isq ? a.oq + row * a.ldoq : a.ok + row * a.ldok) + at;
      float u[N], v[N];
      load_vals<BF16>(g, u);
      load_vals<BF16>(g + D / 2 * E, v);
      if constexpr (NORM) {
        const unsigned char* x = (isq ? a.q + row * a.ldq : a.k + row * a.ldk) + at;
        float x0[N], x1[N];
        load_vals<BF16>(x, x0);
        load_vals<BF16>(x + D / 2 * E, x1);
        turn<PAIRS>(u, v, c, s, -1.f);
        const float* w = isq ? a.wq : a.wk;
        float w0[N], w1[N];
        load_weight(w, j * N, w0);
        load_weight(w, j * N + D / 2, w1);
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          sq += x0[i] * x0[i] + x1[i] * x1[i];
          dot += w0[i] * u[i] * x0[i] + w1[i] * v[i] * x1[i];
        }
        const float r = 1.0f / sqrtf(group_sum<L>(sq) * (1.0f / D) + a.eps);
        const float m = group_sum<L>(dot) * (1.0f / D) * r * r;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float d0 = u[i] * x0[i] * r, d1 = v[i] * x1[i] * r;
          sum[0][i] += isq ? d0 : 0.f;
          sum[0][N + i] += isq ? d1 : 0.f;
          sum[1][i] += isq ? 0.f : d0;
          sum[1][N + i] += isq ? 0.f : d1;
          u[i] = r * (w0[i] * u[i] - x0[i] * m);
          v[i] = r * (w1[i] * v[i] - x1[i] * m);
        }
      } else {
        turn<PAIRS>(u, v, c, s, -1.f);
      }
      store_vals<BF16>(o, u);
      store_vals<BF16>(o + D / 2 * E, v);
    }
  }
  if constexpr (NORM) {
    constexpr int G = kWaves * HPW;   // groups of lanes that hold the same columns
    __shared__ float part[2 * D][G + 1];
    const int grp = (threadIdx.x >> 6) * HPW + hl;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        part[t * D + j * N + i][grp] = sum[t][i];
        part[t * D + D / 2 + j * N + i][grp] = sum[t][N + i];
      }
    __syncthreads();
    for (int col = threadIdx.x; col < 2 * D; col += kThreads) {
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i) v += part[col][i];
      a.partial[(long long)blockIdx.x * (2 * D) + col] = v;
    }
  }
}

// the blocks' partial rows, summed in a fixed order: 64 threads a column, each a
// strided run of the rows, then the 64 in order
__global__ __launch_bounds__(kSumThreads) void rope_sum_kernel(const float* partial, int blocks, int D, float* dwq,
                                                              float* dwk) {
  __shared__ float part[kSumThreads];
  const int c = threadIdx.x % kSumCols, run = threadIdx.x / kSumCols;
  const int col = blockIdx.x * kSumCols + c;   // 2 D is a multiple of kSumCols
  float v = 0.f;
#pragma unroll 16
  for (int b = run; b < blocks; b += kSumThreads / kSumCols) v += partial[(long long)b * (2 * D) + col];
  part[threadIdx.x] = v;
  __syncthreads();
  if (run) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < kSumThreads / kSumCols; ++i) v += part[i * kSumCols + c];
  if (col < D) dwq[col] = v;
  else dwk[col - D] = v;
}

template <bool BACK, bool BF16, int D, bool BATCH>
void launch(const RopeArgs& a, bool pairs, bool norm, int blocks, hipStream_t hs) {
  auto go = [&](auto kern) { kern<<<blocks, kThreads, 0, hs>>>(a); };
  if constexpr (BACK) {
    if (pairs) norm ? go(rope_back_kernel<BF16, D, true, true, BATCH>) : go(rope_back_kernel<BF16, D, true, false, BATCH>);
    else norm ? go(rope_back_kernel<BF16, D, false, true, BATCH>) : go(rope_back_kernel<BF16, D, false, false, BATCH>);
  } else {
    if (pairs) norm ? go(rope_kernel<BF16, D, true, true, BATCH>) : go(rope_kernel<BF16, D, true, false, BATCH>);
    else norm ? go(rope_kernel<BF16, D, false, true, BATCH>) : go(rope_kernel<BF16, D, false, false, BATCH>);
  }
}
template <bool BACK, bool BF16, int D>
void launch(const RopeArgs& a, bool pairs, bool norm, int blocks, hipStream_t hs) {
  if (a.batch) launch<BACK, BF16, D, true>(a, pairs, norm, blocks, hs);
  else launch<BACK, BF16, D, false>(a, pairs, norm, blocks, hs);
}
template <bool BACK>
void launch(const RopeArgs& a, bool bf16, int64_t D, bool pairs, bool norm, int blocks, hipStream_t hs) {
  if (bf16) D == 64 ? launch<BACK, true, 64>(a, pairs, norm, blocks, hs) : launch<BACK, true, 128>(a, pairs, norm, blocks, hs);
  else D == 64 ? launch<BACK, false, 64>(a, pairs, norm, blocks, hs) : launch<BACK, false, 128>(a, pairs, norm, blocks, hs);
}

int back_blocks(int64_t rows) {
  const int64_t b = (rows + kWaves - 1) / kWaves;
  return (int)(b < kMaxBackBlocks ? b : kMaxBackBlocks);
}

dr_status check_sizes(int64_t rows, int64_t T, int Hq, int Hkv, int64_t D, dr_dtype dtype, const float* wq, const float* wk,
                      float eps, const float* table, int64_t table_rows, const int32_t* pos) {
  if (dtype != DR_F32 && dtype != DR_BF16) return DR_ERR_DTYPE;
  if (rows < 0 || Hq < 1 || Hkv < 0 || Hq > 65536 || Hkv > 65536 || D < 1) return DR_ERR_ARG;
  if (!table || table_rows < 1 || !aligned16(table)) return DR_ERR_ARG;
  if (!pos && T < 1) return DR_ERR_ARG;
  if ((wq == nullptr) != (wk == nullptr) || !aligned16(wq) || !aligned16(wk)) return DR_ERR_ARG;
  if (wq && !(eps >= 0.f && eps < 1e30f)) return DR_ERR_ARG;
  if (D != 64 && D != 128) return DR_ERR_UNSUPPORTED;
  // (a workgroup a kWaves rows; a launch takes fewer than 2^32 threads per dimension)
  if (rows > kWaves * (((int64_t)1 << 32) / kThreads - 1)) return DR_ERR_UNSUPPORTED;
  return DR_OK;
}
// one [rows][ld] tensor of H heads
bool good(const void* p, int64_t ld, int64_t H, int64_t D, int64_t rows, dr_dtype dtype) {
  if (rows == 0 || H == 0) return true;
  return p && aligned16(p) && ld >= H * D && ld % (dtype == DR_BF16 ? 8 : 4) == 0;
}

// Takes the layout of b with its N sequences.  Without offsets and lengths every row is a
// token, and the kernels without a lookup run.
dr_status set_batch(RopeArgs& a, const attn::Batch& b, int64_t N) {
  if (N < 0 || b.T < 0) return DR_ERR_ARG;
  if (N > 0x7fffffff || b.T > 0x7fffffff) return DR_ERR_UNSUPPORTED;
  if (b.off ? N == 0 && b.rows > 0 : b.rows != N * b.T) return DR_ERR_ARG;
  a.batch = b.off || b.len;
  a.b = b;
  a.b.N = (int)N;
  a.perT = attn::divisor((unsigned)(b.T > 0 ? b.T : 1));
  return DR_OK;
}

// b, N: NULL without a batch's layout
dr_status forward(const void* q, int64_t ldq, const void* k, int64_t ldk, int64_t rows, int64_t T, const attn::Batch* b,
                  int64_t N, int Hq, int Hkv, int64_t D, dr_dtype dtype, const float* wq, const float* wk, float eps,
                  const float* table, int64_t table_rows, const int32_t* pos, dr_rope_pairing pairing, void* q_out,
                  int64_t ldqo, void* k_out, int64_t ldko, void* stream) {
  const dr_status st = check_sizes(rows, T, Hq, Hkv, D, dtype, wq, wk, eps, table, table_rows, pos);
  if (st != DR_OK) return st;
  if (pairing != DR_ROPE_HALVES && pairing != DR_ROPE_NEIGHBOURS) return DR_ERR_ARG;
  if (!good(q, ldq, Hq, D, rows, dtype) || !good(k, ldk, Hkv, D, rows, dtype) || !good(q_out, ldqo, Hq, D, rows, dtype) ||
      !good(k_out, ldko, Hkv, D, rows, dtype))
    return DR_ERR_ARG;
  RopeArgs a = {};
  const dr_status laid = b ? set_batch(a, *b, N) : DR_OK;
  if (laid != DR_OK || rows == 0) return laid;
  const int e = dtype == DR_BF16 ? 2 : 4;
  a.q = (const unsigned char*)q;
  a.k = (const unsigned char*)k;
  a.oq = (unsigned char*)q_out;
  a.ok = (unsigned char*)k_out;
  a.ldq = ldq * e, a.ldk = ldk * e, a.ldoq = ldqo * e, a.ldok = ldko * e;
  a.rows = rows, a.T = T, a.table_rows = table_rows;
  a.wq = wq, a.wk = wk, a.table = table, a.pos = pos, a.eps = eps;
  a.Hq = Hq, a.H = Hq + Hkv;
  launch<false>(a, dtype == DR_BF16, D, pairing == DR_ROPE_NEIGHBOURS, wq != nullptr, (int)((rows + kWaves - 1) / kWaves),
                (hipStream_t)stream);
  return launch_status();
}

dr_status backward(const void* gq, int64_t ldgq, const void* gk, int64_t ldgk, const void* q, int64_t ldq, const void* k,
                   int64_t ldk, int64_t rows, int64_t T, const attn::Batch* b, int64_t N, int Hq, int Hkv, int64_t D,
                   dr_dtype dtype, const float* wq, const float* wk, float eps, const float* table, int64_t table_rows,
                   const int32_t* pos, dr_rope_pairing pairing, void* dq, int64_t lddq, void* dk, int64_t lddk, float* dwq,
                   float* dwk, void* workspace, size_t ws_bytes, void* stream) {
  const dr_status st = check_sizes(rows, T, Hq, Hkv, D, dtype, wq, wk, eps, table, table_rows, pos);
  if (st != DR_OK) return st;
  if (pairing != DR_ROPE_HALVES && pairing != DR_ROPE_NEIGHBOURS) return DR_ERR_ARG;
  const bool norm = wq != nullptr;
  if (!good(gq, ldgq, Hq, D, rows, dtype) || !good(gk, ldgk, Hkv, D, rows, dtype) || !good(dq, lddq, Hq, D, rows, dtype) ||
      !good(dk, lddk, Hkv, D, rows, dtype))
    return DR_ERR_ARG;
  if (norm && (!good(q, ldq, Hq, D, rows, dtype) || !good(k, ldk, Hkv, D, rows, dtype) || !dwq || !dwk)) return DR_ERR_ARG;
  RopeArgs a = {};
  const dr_status laid = b ? set_batch(a, *b, N) : DR_OK;
  if (laid != DR_OK || (rows == 0 && !norm)) return laid;
  if (norm && rows > 0 && (!workspace || ws_bytes < dr_qk_norm_rope_workspace_size(rows, D))) return DR_ERR_WORKSPACE;
  const int e = dtype == DR_BF16 ? 2 : 4;
  a.gq = (const unsigned char*)gq;
  a.gk = (const unsigned char*)gk;
  a.q = (const unsigned char*)q;
  a.k = (const unsigned char*)k;
  a.oq = (unsigned char*)dq;
  a.ok = (unsigned char*)dk;
  a.ldgq = ldgq * e, a.ldgk = ldgk * e, a.ldq = ldq * e, a.ldk = ldk * e, a.ldoq = lddq * e, a.ldok = lddk * e;
  a.rows = rows, a.T = T, a.table_rows = table_rows;
  a.wq = wq, a.wk = wk, a.table = table, a.pos = pos, a.eps = eps;
  a.Hq = Hq, a.H = Hq + Hkv;
  a.partial = (float*)workspace;
  const hipStream_t hs = (hipStream_t)stream;
  const int blocks = rows > 0 ? back_blocks(rows) : 0;
  if (rows > 0) launch<true>(a, dtype == DR_BF16, D, pairing == DR_ROPE_NEIGHBOURS, norm, blocks, hs);
  if (norm)   // (no rows: writes zeros)
    rope_sum_kernel<<<(int)(2 * D / kSumCols), kSumThreads, 0, hs>>>(a.partial, blocks, (int)D, dwq, dwk);
  return launch_status();
}

}  // namespace
}  // namespace dr

extern "C" dr_status dr_qk_norm_rope(const void* q, int64_t ldq, const void* k, int64_t ldk, int64_t rows, int64_t T, int Hq,
                                     int Hkv, int64_t D, dr_dtype dtype, const float* wq, const float* wk, float eps,
                                     const float* table, int64_t table_rows, const int32_t* pos, dr_rope_pairing pairing,
                                     void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream) {
  return dr::forward(q, ldq, k, ldk, rows, T, nullptr, 0, Hq, Hkv, D, dtype, wq, wk, eps, table, table_rows, pos, pairing,
                     q_out, ldqo, k_out, ldko, stream);
}

extern "C" dr_status dr_qk_norm_rope_batch(const void* q, int64_t ldq, const void* k, int64_t ldk, int64_t rows, int64_t N,
                                           int64_t T, const int32_t* off, const int32_t* len, int Hq, int Hkv, int64_t D,
                                           dr_dtype dtype, const float* wq, const float* wk, float eps, const float* table,
                                           int64_t table_rows, const int32_t* pos, dr_rope_pairing pairing, void* q_out,
                                           int64_t ldqo, void* k_out, int64_t ldko, void* stream) {
  const dr::attn::Batch b = {off, len, rows, T, 0};
  return dr::forward(q, ldq, k, ldk, rows, T > 0 ? T : 1, &b, N, Hq, Hkv, D, dtype, wq, wk, eps, table, table_rows, pos,
                     pairing, q_out, ldqo, k_out, ldko, stream);
}

extern "C" size_t dr_qk_norm_rope_workspace_size(int64_t rows, int64_t D) {
  if (rows < 1 || D < 1) return 0;
  return (size_t)dr::back_blocks(rows) * 2 * (size_t)D * sizeof(float);
}

extern "C" dr_status dr_qk_norm_rope_backward(const void* gq, int64_t ldgq, const void* gk, int64_t ldgk, const void* q,
                                              int64_t ldq, const void* k, int64_t ldk, int64_t rows, int64_t T, int Hq,
                                              int Hkv, int64_t D, dr_dtype dtype, const float* wq, const float* wk, float eps,
                                              const float* table, int64_t table_rows, const int32_t* pos,
                                              dr_rope_pairing pairing, void* dq, int64_t lddq, void* dk, int64_t lddk,
                                              float* dwq, float* dwk, void* workspace, size_t ws_bytes, void* stream) {
  return dr::backward(gq, ldgq, gk, ldgk, q, ldq, k, ldk, rows, T, nullptr, 0, Hq, Hkv, D, dtype, wq, wk, eps, table,
                      table_rows, pos, pairing, dq, lddq, dk, lddk, dwq, dwk, workspace, ws_bytes, stream);
}

extern "C" dr_status dr_qk_norm_rope_batch_backward(
    const void* gq, int64_t ldgq, const void* gk, int64_t ldgk, const void* q, int64_t ldq, const void* k, int64_t ldk,
    int64_t rows, int64_t N, int64_t T, const int32_t* off, const int32_t* len, int Hq, int Hkv, int64_t D, dr_dtype dtype,
    const float* wq, const float* wk, float eps, const float* table, int64_t table_rows, const int32_t* pos,
    dr_rope_pairing pairing, void* dq, int64_t lddq, void* dk, int64_t lddk, float* dwq, float* dwk, void* workspace,
    size_t ws_bytes, void* stream) {
  const dr::attn::Batch b = {off, len, rows, T, 0};
  return dr::backward(gq, ldgq, gk, ldgk, q, ldq, k, ldk, rows, T > 0 ? T : 1, &b, N, Hq, Hkv, D, dtype, wq, wk, eps, table,
                      table_rows, pos, pairing, dq, lddq, dk, lddk, dwq, dwk, workspace, ws_bytes, stream);
}

// What the attention kernels over the 4-bit cache share: how the work is cut, who sees what, how pieces are joined.
//
// The work is a line of steps (a few blocks of one head for one tile of query rows): requests, then kv heads, then tiles of
// rows, then steps.  A unit = the steps of one (request, head, tile), behind a lead that stands for what a unit costs besides
// (queries, results).  The line is cut into equal pieces, one a CTA, whatever the lengths of the contexts are (they are known on the
// device only).  A unit that lies within one CTA is written by it; the pieces of another go to the workspace, with a record by
// which the join kernel finds them.
#pragma once

#include "ts_cache.cuh"

namespace ts {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttnArgs {
  CacheDims d;
  int B, rcap, N, words;   // rows a request has room for; nodes and mask words of the context
  const void* q; long long ldq;
  const unsigned char* pool;
  const int *table, *seq_len, *n_nodes;
  const uint64_t* mask;
  unsigned by_g;           // ceil(2^32 / G): idx * by_g >> 32 = idx / G for all idx below 2^19 and G up to 1,024
  float qk, vo;            // powers of two of the operands, the scale and log2 e; what takes V's power of two back
  void* out; long long ldo;
  float* lse;
  struct AttnRecord* records; float* part; float* part_ml;   // workspace: [grid], [grid][2][QT][Dh], [grid][2][QT][2]
  int grid;                // CTAs at most
  int min_steps;           // steps that make a piece worth a CTA of its own
  unsigned limit;          // polls before a wait gives up
  unsigned lost;           // bytes that the waits for copies expect and that do not come (0 but in the library's own tests)
};

// pieces first..last of a unit; first < 0: nothing begins here that is to be joined
struct AttnRecord { int b, v, first, last, nq, rows; };

// v = head * nq + tile; n steps behind the lead, which begins at place t0
struct AttnUnit { int b, v, n, nq, rows, seq; long long t0; };

// QT query rows a tile, TOK tokens a step; a lead is as long as LEAD steps
template <int QT_, int TOK_, int LEAD_>
struct AttnShape {
  static constexpr int QT = QT_, TOK = TOK_, LEAD = LEAD_;
};

// the request's units: fills all of u but v and t0; returns how many there are
template <class S>
__device__ __forceinline__ int unit_set(const AttnArgs& a, int b, AttnUnit& u) {
  u.b = b; u.seq = a.seq_len[b];
  u.rows = request_rows(a.n_nodes, b, a.rcap);
  if (u.seq < 0) { u.n = 0; u.nq = 0; return 0; }
  const unsigned end = min((unsigned)u.seq + (unsigned)u.rows, (unsigned)a.d.cols * (unsigned)a.d.ps);   // (no page beyond the table's)
  u.n = max(1u, (end + S::TOK - 1) / S::TOK);
  u.nq = (u.rows * a.d.G + S::QT - 1) / S::QT;
  return a.d.Hkv * u.nq;
}

// (a division of 64 bits is a call of a hundred instructions; almost all of these fit 32)
__device__ __forceinline__ long long divide(long long x, long long y) { return (unsigned long long)(x | y) >> 32 ? x / y : (long long)((unsigned)x / (unsigned)y); }

// CTAs that take part, where piece c begins, and the piece in which place x lies
__device__ __forceinline__ int attn_active(const AttnArgs& a, long long total) { return (int)min((long long)a.grid, max(1ll, divide(total, a.min_steps))); }
__device__ __forceinline__ long long piece_start(long long total, int active, int c) { return divide(total * c, active); }
__device__ __forceinline__ int piece_of(long long total, int active, long long x) { return (int)divide((x + 1) * active + total - 1, total) - 1; }

// (to be called where there is one)
template <class S>
__device__ __forceinline__ void next_unit(const AttnArgs& a, AttnUnit& u) {
  u.t0 += u.n + S::LEAD;
  if (++u.v >= a.d.Hkv * u.nq) {
    u.v = 0;
    for (int b = u.b + 1; b < a.B; ++b)
      if (unit_set<S>(a, b, u) > 0) break;
  }
}

// Finds this CTA's steps: the unit of the first, its number there, and how many there are.  All threads call it; false: none.
template <class S, int THREADS>
__device__ bool attn_locate(const AttnArgs& a, AttnUnit& u, int& first, long long& steps) {
  __shared__ long long wsum[THREADS / 32][2], before[2];   // before: steps before the piece's beginning and end
  __shared__ AttnUnit found;
  __shared__ int found_step;
  const int per = (a.B + THREADS - 1) / THREADS, b0 = threadIdx.x * per, b1 = min(b0 + per, a.B), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long sum = 0, cnt = 0;   // length and steps of this thread's requests
  for (int b = b0; b < b1; ++b) {
    const long long units = unit_set<S>(a, b, u);
    sum += units * (u.n + S::LEAD);
    cnt += units * u.n;
  }
  long long at = sum, nth = cnt;
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(~0u, at, o), y = __shfl_up_sync(~0u, nth, o);
    if (lane >= o) { at += x; nth += y; }
  }
  if (lane == 31) { wsum[warp][0] = at; wsum[warp][1] = nth; }
  at -= sum; nth -= cnt;
  __syncthreads();
  long long total = 0, all = 0;
  const int warps = min(THREADS / 32, (a.B + 32 * per - 1) / (32 * per));   // that have requests
#pragma unroll 1
  for (int w = 0; w < warps; ++w) {
    if (w < warp) { at += wsum[w][0]; nth += wsum[w][1]; }
    total += wsum[w][0]; all += wsum[w][1];
  }
  const int active = attn_active(a, total);
  if (total == 0 || (int)blockIdx.x >= active) {
    if (threadIdx.x == 0) a.records[blockIdx.x].first = -1;
    return false;
  }
  const long long x0 = piece_start(total, active, blockIdx.x), x1 = piece_start(total, active, blockIdx.x + 1);
  if (threadIdx.x == 0 && x1 == total) before[1] = all;
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    long long x = (side ? x1 : x0) - at, k = nth;
    if (x < 0 || x >= sum) continue;
    for (int b = b0;; ++b) {
      const long long units = per == 1 ? (long long)a.d.Hkv * u.nq : unit_set<S>(a, b, u), len = u.n + S::LEAD;   // (one request a thread: u has it)
      if (x < units * len) {
        u.v = (int)divide(x, len);
        x -= u.v * len;   // within the unit
        u.t0 = (side ? x1 : x0) - x;
        const int j = (int)max(x - S::LEAD, 0ll);   // the first step that begins there or later
        before[side] = k + (long long)u.v * u.n + j;
        if (side == 0) { found = u; found_step = j; }
        break;
      }
      x -= units * len;
      k += units * u.n;
    }
  }
  __syncthreads();
  u = found;
  first = found_step;
  steps = before[1] - before[0];
  if (threadIdx.x == 0) {
    // the first cut between steps of the unit: the piece before this one holds its beginning
    AttnRecord r{u.b, u.v, -1, 0, u.nq, u.rows};
    const long long step0 = u.t0 + S::LEAD;
    if (steps > 0 && first > 0 && piece_of(total, active, step0) == (int)blockIdx.x - 1) {
      r.first = blockIdx.x - 1;
      r.last = piece_of(total, active, step0 + u.n - 1);
    }
    a.records[blockIdx.x] = r;
  }
  return steps > 0;
}

// Whether tree row i of request b sees the token at place rel behind the prefix (rel >= 0).
__device__ __forceinline__ bool row_sees(const AttnArgs& a, int b, int i, int rel, int rows) {
  if (rel >= rows || i >= rows) return false;
  if (!a.mask) return rel <= i;
  if (rel == 0) return true;
  if (i == 0) return false;
  return (a.mask[((size_t)b * a.N + (i - 1)) * a.words + ((rel - 1) >> 6)] >> ((rel - 1) & 63)) & 1ull;
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float lg2(float x) {
  float r;
  asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// the tree row of row idx of a kv head, and where that row goes
__device__ __forceinline__ int tree_row(const AttnArgs& a, int idx) { return a.d.G == 1 ? idx : (int)__umulhi((unsigned)idx, a.by_g); }
__device__ __forceinline__ size_t head_row(const AttnArgs& a, int b, int h, int idx, long long ld) {
  const int i = tree_row(a, idx);
  return ((size_t)b * a.rcap + i) * ld + (size_t)(h * a.d.G + idx - i * a.d.G) * a.d.Dh;
}
__device__ __forceinline__ size_t out_row(const AttnArgs& a, int b, int h, int idx) { return head_row(a, b, h, idx, a.ldo); }
__device__ __forceinline__ size_t lse_row(const AttnArgs& a, int b, int h, int idx) {
  const int i = tree_row(a, idx);
  return ((size_t)b * a.rcap + i) * a.d.Hq + h * a.d.G + idx - i * a.d.G;
}

// A row's weight sum l relative to 2^m, as the natural logarithm of the row's sum.  No token: l = 0.
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + lg2(l)) * LN2; }
__device__ __forceinline__ float row_inv(float l) { return l == 0.f ? 0.f : 1.f / l; }
// what a part of a row counts in the whole; a part that has seen nothing counts zero (a NaN in it stays one)
__device__ __forceinline__ float part_weight(float m, float top) { return m == -INFINITY ? 0.f : ex2(m - top); }

// the workspace of a launch, and where its parts lie
size_t attn_workspace(int grid, int QT, int Dh);
void attn_place(AttnArgs& a, int QT, char* ws);
cudaError_t attn_join(ts_ctx* ctx, const AttnArgs& a, int QT, bool f32, cudaStream_t st);
// many query rows a kv head (ts_attn_many.cu), bf16 only
cudaError_t attn_many_setup(ts_ctx* ctx);
size_t attn_many_workspace(const ts_ctx* ctx, const CacheDims& d);
cudaError_t attn_many_launch(ts_ctx* ctx, AttnArgs a, char* ws, cudaStream_t st);

}  // namespace ts

// What the attention kernels over the 4-bit cache share: how the work is cut, who sees what, how pieces are joined.
//
// The work is a line of steps (a few blocks of one head for one tile of query rows): requests, then kv heads, then tiles of
// rows, then steps.  A unit = the steps of one (request, head, tile).  The line is cut into equal pieces, one a CTA,
// whatever the lengths are: lengths are known on the device only.  A unit that lies within one CTA is written by it; the
// pieces of another go to the workspace, with a record by which the join kernel finds them.
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
  float qk, vo;            // powers of two of the operands, the scale and log2 e; what takes V's power of two back
  void* out; long long ldo;
  float* lse;
  struct AttnRecord* records; float* part; float* part_ml;   // workspace: [grid], [grid][2][QT][Dh], [grid][2][QT][2]
  int grid;                // CTAs at most
  int min_steps;           // steps that make a piece worth a CTA of its own
  unsigned limit;          // polls before a wait gives up
};

// pieces first..last of a unit; first < 0: nothing begins here that is to be joined
struct AttnRecord { int b, v, first, last; long long t0; int nq, active; };

struct AttnUnit { int b, v, n, nq, rows, seq; long long t0; };   // v = head * nq + tile; n steps, the first at place t0

// QT query rows a tile, TOK tokens a step
template <int QT, int TOK>
__device__ __forceinline__ long long unit_steps(const AttnArgs& a, int b, AttnUnit& u) {
  u.b = b; u.seq = a.seq_len[b];
  u.rows = request_rows(a.n_nodes, b, a.rcap);
  if (u.seq < 0) { u.n = 0; u.nq = 0; return 0; }
  const long long end = min((long long)u.seq + u.rows, (long long)a.d.cols * a.d.ps);   // (no page beyond the table's)
  u.n = (int)max(1ll, (end + TOK - 1) / TOK);
  u.nq = (u.rows * a.d.G + QT - 1) / QT;
  return (long long)a.d.Hkv * u.nq * u.n;
}

// CTAs that take part, and where piece c begins
__device__ __forceinline__ int attn_active(const AttnArgs& a, long long total) { return (int)min((long long)a.grid, max(1ll, total / a.min_steps)); }
__device__ __forceinline__ long long piece_start(long long total, int active, int c) { return total * c / active; }

template <int QT, int TOK>
__device__ __forceinline__ void next_unit(const AttnArgs& a, AttnUnit& u) {
  u.t0 += u.n;
  if (++u.v < a.d.Hkv * u.nq) return;
  u.v = 0;
  while (++u.b < a.B) {
    AttnUnit n = u;
    if (unit_steps<QT, TOK>(a, u.b, n) > 0) { n.t0 = u.t0; n.v = 0; u = n; return; }
  }
}

// Finds the whole line's length and the unit in which this CTA's piece begins.  All threads call it; false: no piece.
template <int QT, int TOK, int THREADS>
__device__ bool attn_locate(const AttnArgs& a, AttnUnit& u, long long& start, long long& end, int& active) {
  __shared__ long long wsum[THREADS / 32];
  __shared__ AttnUnit found;
  const int per = (a.B + THREADS - 1) / THREADS, b0 = threadIdx.x * per, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  AttnUnit n;
  long long sum = 0;
  for (int b = b0; b < min(b0 + per, a.B); ++b) sum += unit_steps<QT, TOK>(a, b, n);
  long long inc = sum;
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(~0u, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) wsum[warp] = inc;
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += wsum[w];
    total += wsum[w];
  }
  active = attn_active(a, total);
  if (total == 0 || (int)blockIdx.x >= active) {
    if (threadIdx.x == 0) a.records[blockIdx.x].first = -1;
    return false;
  }
  start = piece_start(total, active, blockIdx.x);
  end = piece_start(total, active, blockIdx.x + 1);
  long long at = before + inc - sum;
  if (start >= at && start < at + sum)
    for (int b = b0;; ++b) {
      const long long w = unit_steps<QT, TOK>(a, b, n);
      if (start < at + w) {
        n.v = (int)((start - at) / n.n);
        n.t0 = at + (long long)n.v * n.n;
        found = n;
        break;
      }
      at += w;
    }
  __syncthreads();
  u = found;
  if (threadIdx.x == 0) {
    // the first cut within the unit: the piece before this one holds its beginning
    AttnRecord r{u.b, u.v, -1, 0, u.t0, u.nq, active};
    if (start > u.t0 && piece_start(total, active, blockIdx.x - 1) <= u.t0) {
      r.first = blockIdx.x - 1;
      r.last = (int)(((u.t0 + u.n) * active + total - 1) / total) - 1;   // the last c with start(c) < end of the unit
    }
    a.records[blockIdx.x] = r;
  }
  return true;
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

// where row idx of a request's head goes
__device__ __forceinline__ size_t out_row(const AttnArgs& a, int b, int h, int idx) { return ((size_t)b * a.rcap + idx / a.d.G) * a.ldo + (size_t)(h * a.d.G + idx % a.d.G) * a.d.Dh; }
__device__ __forceinline__ size_t lse_row(const AttnArgs& a, int b, int h, int idx) { return ((size_t)b * a.rcap + idx / a.d.G) * a.d.Hq + h * a.d.G + idx % a.d.G; }

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

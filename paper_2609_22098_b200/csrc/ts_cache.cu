// The 4-bit cache around the attention: pages and slots for a round's rows (reserve), keys and values into their slots
// (append), the accepted path's rows to the end of the prefix (commit).
#include "ts_cache.cuh"

#include <algorithm>
#include <stdio.h>

#include <cooperative_groups.h>

namespace ts {

const char* cache_layout_error(const ts_cache_layout* l) {
  if (!l) return "null layout";
  if (l->Hq < 1 || l->Hkv < 1 || l->Hq % l->Hkv != 0 || l->Hq > 1024) return "Hq must be a multiple of Hkv, at most 1024";
  if (l->Dh != 64 && l->Dh != 128) return "head size must be 64 or 128";
  if (l->page_size < CACHE_BLOCK || l->page_size % CACHE_BLOCK || l->page_size > 4096) return "page size must be a multiple of 16, at most 4096";
  if (l->n_pages < 1 || l->max_pages < 1) return "sizes must be positive";
  if ((long long)l->n_pages * l->page_size > 0x7FFFFFFFll || (long long)l->max_pages * l->page_size > 0x7FFFFFFFll) return "more than 2^31 - 1 slots or positions";
  if (l->dtype != TS_DTYPE_F32 && l->dtype != TS_DTYPE_BF16) return "dtype must be f32 or bf16";
  if (l->k_exp < -30 || l->k_exp > 30 || l->v_exp < -30 || l->v_exp > 30) return "exponents must lie in -30..30";
  return nullptr;
}

int32_t set_layout_error(const char* call, const ts_cache_layout* l) {
  char msg[256];
  snprintf(msg, sizeof(msg), "%s: %s", call, cache_layout_error(l));
  return set_error(l ? TS_ERR_UNSUPPORTED : TS_ERR_INVALID, msg);
}

CacheDims cache_dims(const ts_cache_layout* l) {
  CacheDims d;
  d.Hq = l->Hq; d.Hkv = l->Hkv; d.G = l->Hq / l->Hkv; d.Dh = l->Dh; d.ps = l->page_size; d.n_pages = l->n_pages; d.cols = l->max_pages;
  return d;
}

bool on_ctx_device(const ts_ctx* ctx) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->device;
}

// ------------------------------------------------------------------------------------------------
// Reserve.  Every CTA adds up the pages that all requests need (a few thousand at most), then serves its share of the
// requests, one warp each (and all of its warps for the many entries of a request that starts).  Small calls are one launch of a
// cluster of eight CTAs whose barrier separates reading the counts from writing them, so that they may be updated in place;
// where whole tables are written, many CTAs write them and a second launch updates the counts.  Bound by latency (counts, a scan, entries,
// slots and two barriers one after the other): a round of 32 requests moves 9 KB in 5.4 us, 500 requests that start with tables of
// up to 1,875 entries move 3.8 MB in 10.0.
// ------------------------------------------------------------------------------------------------
constexpr int RES_THREADS = 512;
constexpr int RES_CLUSTER = 8;
constexpr int RES_MAX_B = 4096;
// The cluster's form: up to this many requests and table entries (requests times columns, what the host knows).  A round of 32
// requests with 500 columns takes the cluster 5.2 us and many CTAs 6.4 (and the host a second launch), 32 whole tables of 500
// columns 7.1 and 6.6, of 2,000 columns 8.9 and 7.5, 128 of 500 columns 15 and 6.8, 500 of 1,875 columns 77 and 10.
constexpr int RES_CLUSTER_B = 64;
constexpr long long RES_CLUSTER_ENTRIES = 1 << 16;

struct ReserveArgs {
  CacheDims d;
  int B, rcap;
  const int *seq_len, *n_nodes, *held, *free_count;
  int *free_pages, *table, *held_out, *free_count_out, *slot_map, *status;
};

struct ReservePlan { int rows, held, need, start; bool granted, release; };

// pages needed by request b; -1: it gives its pages back
__device__ __forceinline__ int pages_needed(const ReserveArgs& a, int b) {
  const int n = a.seq_len[b];
  if (n < 0) return -1;
  const unsigned end = (unsigned)n + (unsigned)request_rows(a.n_nodes, b, a.rcap);   // below 2^31 + 257
  const unsigned need = (end + (unsigned)a.d.ps - 1u) / (unsigned)a.d.ps;           // (a division of 64 bits is a call)
  return need > (unsigned)a.d.cols ? a.d.cols + 1 : (int)need;
}
__device__ __forceinline__ int pages_held(const ReserveArgs& a, int b) { return min(max(a.held[b], 0), a.d.cols); }
__device__ __forceinline__ int pages_taken(const ReserveArgs& a, int b) {
  const int need = pages_needed(a, b);
  return need < 0 || need > a.d.cols ? 0 : max(0, need - pages_held(a, b));
}

// pages taken (low half) and entries given back (high half); each half stops at 2^31 - 1, which is more than a pool has pages
__device__ __forceinline__ long long pages_of(const ReserveArgs& a, int b) {
  return (long long)pages_taken(a, b) + (a.seq_len[b] < 0 ? (long long)pages_held(a, b) << 32 : 0ll);
}
__device__ __forceinline__ long long add_pages(long long x, long long y) {
  const unsigned top = 0x7FFFFFFFu;
  return (long long)((unsigned long long)min((unsigned)(x >> 32) + (unsigned)(y >> 32), top) << 32 | min((unsigned)x + (unsigned)y, top));
}

// Exclusive running sums over requests of what `of` says, in shared memory (where `of` may look for its own request); returns the total.
template <class Of>
__device__ long long reserve_scan(int B, long long* pre, Of of) {
  __shared__ long long wsum[RES_THREADS / 32];
  const int per = (B + RES_THREADS - 1) / RES_THREADS, b0 = threadIdx.x * per, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long sum = 0;
  for (int b = b0; b < min(b0 + per, B); ++b) sum = add_pages(sum, pre[b] = of(b));
  long long inc = sum;
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(~0u, inc, o);
    if (lane >= o) inc = add_pages(inc, v);
  }
  if (lane == 31) wsum[warp] = inc;
  long long at = __shfl_up_sync(~0u, inc, 1);
  if (lane == 0) at = 0;
  __syncthreads();
  long long all = 0;
  for (int w = 0; w < RES_THREADS / 32; ++w) {
    if (w < warp) at = add_pages(wsum[w], at);
    all = add_pages(all, wsum[w]);
  }
  for (int b = b0; b < min(b0 + per, B); ++b) {
    const long long mine = pre[b];
    pre[b] = at;
    at = add_pages(at, mine);
  }
  __syncthreads();
  return all;
}

__device__ __forceinline__ ReservePlan plan_of(const ReserveArgs& a, int b, long long pre, int count) {
  ReservePlan p;
  p.rows = request_rows(a.n_nodes, b, a.rcap);
  p.held = pages_held(a, b);
  p.need = pages_needed(a, b);
  p.release = p.need < 0;
  p.start = (int)(pre & 0xFFFFFFFFll);
  const int take = p.need > a.d.cols ? 0 : max(0, p.need - p.held);
  p.granted = !p.release && p.need <= a.d.cols && (take == 0 || (long long)p.start + take <= count);
  return p;
}

// one warp: the slots of a request's rows and its new table entries, or the first of them where they are many
constexpr int RES_SHORT = 64;   // entries of a request that its warp writes; what is more is written by the whole CTA
__device__ void reserve_rows(const ReserveArgs& a, int b, const ReservePlan& p, int count, int lane) {
  int* row = a.table + (size_t)b * a.d.cols;
  if (p.granted)
    for (int c = p.held + lane; c < min(p.need, p.held + RES_SHORT); c += 32) row[c] = a.free_pages[count - 1 - (p.start + c - p.held)];
  const int first = a.seq_len[b];
  for (int i = lane; i < a.rcap; i += 32) {
    int slot = -1;
    if (p.granted && i < p.rows) {
      const int pos = first + i, c = (unsigned)pos / (unsigned)a.d.ps;
      const int page = c < p.held ? row[c] : a.free_pages[count - 1 - (p.start + c - p.held)];
      if ((unsigned)page < (unsigned)a.d.n_pages) slot = page * a.d.ps + (pos - c * a.d.ps);
    }
    a.slot_map[(size_t)b * a.rcap + i] = slot;
  }
  if (lane == 0) a.status[b] = p.release || p.granted ? TS_OK : TS_ERR_OVERFLOW;
}

// a CTA's requests (every gridDim.x-th): a warp each, then the long ones by all threads
__device__ void reserve_tables(const ReserveArgs& a, const long long* pre, int count) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = gridDim.x;
  for (int b = blockIdx.x + warp * step; b < a.B; b += RES_THREADS / 32 * step) reserve_rows(a, b, plan_of(a, b, pre[b], count), count, lane);
  if (a.d.cols <= RES_SHORT) return;
  for (int b = blockIdx.x; b < a.B; b += step) {
    if (pages_taken(a, b) <= RES_SHORT) continue;
    const ReservePlan p = plan_of(a, b, pre[b], count);
    if (!p.granted) continue;
    int* row = a.table + (size_t)b * a.d.cols;
#pragma unroll 4
    for (int c = p.held + RES_SHORT + threadIdx.x; c < p.need; c += RES_THREADS) row[c] = a.free_pages[count - 1 - (p.start + c - p.held)];
  }
}

// The last request that got pages ends at this many (the running sum does not fall, so those that got some come first).
__device__ int reserve_taken(const ReserveArgs& a, const long long* pre, int count) {
  __shared__ int top;
  if (threadIdx.x == 0) top = 0;
  __syncthreads();
  int best = 0;
  for (int b = threadIdx.x; b < a.B; b += RES_THREADS) {
    const ReservePlan p = plan_of(a, b, pre[b], count);
    // (one that takes nothing stands at a running sum that may count refused requests before it)
    if (p.granted && p.need > p.held) best = max(best, p.start + p.need - p.held);
  }
  atomicMax(&top, best);
  __syncthreads();
  return top;
}

// WHERE 0: everything, by one cluster; 1: tables and slots; 2: the counts and the pages given back, by one CTA after 1.  (One CTA an SM in
// the bounds: the compiler takes 32 registers otherwise and spills; a round of 32 requests 5.6 and 5.4 us.)
template <int WHERE>
__global__ void __launch_bounds__(RES_THREADS, 1) reserve_kernel(const ReserveArgs a) {
  extern __shared__ long long pre[];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int count = min(max(a.free_count[0], 0), a.d.n_pages);
  const long long all = reserve_scan(a.B, pre, [&](int b) { return pages_of(a, b); });
  if (WHERE == 2 || WHERE == 0) {
    const int taken = reserve_taken(a, pre, count);
    // the plans of this thread's requests, before anything is written in place
    constexpr int OWN = RES_MAX_B / RES_THREADS;
    int new_held[OWN];
    const int warps = (WHERE == 0 ? RES_CLUSTER : 1) * (RES_THREADS / 32), me = blockIdx.x * (RES_THREADS / 32) + (threadIdx.x >> 5);
    if (WHERE == 0) reserve_tables(a, pre, count);
    if (blockIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        const int b = threadIdx.x + k * RES_THREADS;
        if (b >= a.B) break;
        const ReservePlan p = plan_of(a, b, pre[b], count);
        new_held[k] = p.release ? 0 : p.granted ? max(p.held, p.need) : p.held;
      }
    }
    // Entries that are pages, of the requests that give theirs back: what else stands in a table does not go on the list.  (Every CTA
    // counts all of them, and before any of them is overwritten.)
    const bool gives = all >> 32 != 0;   // (the same in all CTAs)
    long long back = 0;
    if (gives) {
      __syncthreads();   // the sums of taken pages are not needed any more
      for (int b = threadIdx.x >> 5; b < a.B; b += RES_THREADS / 32) {
        int n = 0;
        if (a.seq_len[b] < 0) {
          const int held = pages_held(a, b);
          const int* row = a.table + (size_t)b * a.d.cols;
#pragma unroll 4
          for (int c = lane; c < held; c += 32) n += (unsigned)row[c] < (unsigned)a.d.n_pages;
        }
        n = __reduce_add_sync(~0u, n);
        if (lane == 0) pre[b] = n;
      }
      __syncthreads();
      back = reserve_scan(a.B, pre, [&](int b) { return pre[b]; });
    }
    // Given-back pages go where the taken ones lay: every CTA has read those by now.
    const int base = count - taken;
    if (WHERE == 0) cooperative_groups::this_cluster().sync();
    else __syncthreads();
    for (int b = me; gives && b < a.B; b += warps) {
      if (a.seq_len[b] >= 0) continue;
      // (held[b] may be written by CTA 0 below once all have passed the second barrier only)
      const int n = pages_held(a, b);
      long long at = base + pre[b];   // (in 64 bits: a table may name a page twice)
      int* row = a.table + (size_t)b * a.d.cols;
#pragma unroll 4
      for (int c0 = 0; c0 < n; c0 += 32) {
        const int c = c0 + lane, page = c < n ? row[c] : -1;
        const bool is_page = (unsigned)page < (unsigned)a.d.n_pages;
        const unsigned are = __ballot_sync(~0u, is_page);
        const long long to = at + __popc(are & ((1u << lane) - 1u));
        if (c < n) row[c] = -1;
        if (is_page && to < a.d.n_pages) a.free_pages[to] = page;
        at += __popc(are);
      }
    }
    if (gives) {
      if (WHERE == 0) cooperative_groups::this_cluster().sync();
      else __syncthreads();
    }
    if (blockIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        const int b = threadIdx.x + k * RES_THREADS;
        if (b >= a.B) break;
        a.held_out[b] = new_held[k];
      }
      if (threadIdx.x == 0) a.free_count_out[0] = (int)min(base + back, (long long)a.d.n_pages);
    }
  } else {
    reserve_tables(a, pre, count);
  }
}

static cudaError_t launch_reserve(ts_ctx* ctx, const ReserveArgs& a, cudaStream_t st) {
  const size_t smem = (size_t)a.B * sizeof(long long);
  if (a.B <= RES_CLUSTER_B && (long long)a.B * a.d.cols <= RES_CLUSTER_ENTRIES) {
    ProfScope ps(ctx, K_RESERVE, st);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(RES_CLUSTER); cfg.blockDim = dim3(RES_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = RES_CLUSTER; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, reserve_kernel<0>, a);
  }
  cudaError_t e;
  {
    ProfScope ps(ctx, K_RESERVE, st);
    const int grid = std::min(a.B, 2 * ctx->num_sms);
    e = launch_kernel(reserve_kernel<1>, dim3(grid), dim3(RES_THREADS), smem, st, true, a);
  }
  if (e != cudaSuccess) return e;
  ProfScope ps(ctx, K_RESERVE, st);
  return launch_kernel(reserve_kernel<2>, dim3(1), dim3(RES_THREADS), smem, st, true, a);
}

// ------------------------------------------------------------------------------------------------
// Append.  A lane takes eight elements of a row's head (two lanes share a scale), Dh/4 lanes both K and V of one (row, head),
// so that what is not finite in either marks both.  Chunks of 64 requests (102 to 257 rows each, 4 heads of 64 channels, fp32, with
// values): 12.4 us on the device for 50 MB, 4 TB/s; the trees of 32 requests in bf16 6.7 us for 11 MB.  Bound by issue (74 % of the slots while
// SMs are active) and by the ramp of so short a kernel (they are for 71 % of it); two rows a lane, side by side, took as long.
// ------------------------------------------------------------------------------------------------
constexpr int APP_THREADS = 128;   // (128, 256, 512: the chunks below take 12.8, 13.1, 14.5 us in a row)

struct AppendArgs {
  CacheDims d;
  long long items;     // rows * Hkv
  long long ldk, ldv;  // elements between rows
  const void *k, *v;
  const int* slot_map;
  unsigned char* pool;
  void *k_val, *v_val;
  int k_exp, v_exp;
};

__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* x) { unpack_bf16x8(__ldg(reinterpret_cast<const uint4*>(p)), x); }
__device__ __forceinline__ void store8(float* p, const float* x) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// WHOLE + x / s to the nearest whole number, the even one of two as near, without a division or a conversion (which run at a
// quarter of the rate): at 1.5 * 2^23 a sum is rounded to whole numbers, and the number stands in its last bits.  The product
// with 1/s is off by 2^-23 of it, so what it is rounded to is the result or next to it; what is left of x says which, exactly,
// because it is a multiple of x's last place and no larger than x.  (Beyond 2^22 the sum is no whole number apart, and no matter:
// codes end at 7.)
constexpr float WHOLE = 12582912.f;
__device__ __forceinline__ float nearest_code(float x, float s, float inv) {
  float t = fmaf(x, inv, WHOLE);
  const float r = fmaf(WHOLE - t, s, x);
  // more than half of s is left, or just half and the number is odd: magnitudes compare as integers
  const unsigned left = __float_as_uint(r) & 0x7FFFFFFFu, odd = __float_as_uint(t) & 1u;
  if (left + odd > __float_as_uint(0.5f * s)) t += copysignf(1.f, r);
  return fminf(fmaxf(t, WHOLE - 8.f), WHOLE + 7.f);
}

template <typename T, int Dh>
__global__ void __launch_bounds__(APP_THREADS) append_kernel(const AppendArgs a) {
  constexpr int LANES = Dh / 4;             // 32 or 16 lanes a (row, head): the first half K, the second V
  pdl_wait();
  pdl_launch_dependents();
  const long long item = ((long long)blockIdx.x * APP_THREADS + threadIdx.x) / LANES;
  const int l = threadIdx.x % LANES;
  const bool is_v = l >= LANES / 2;
  const int c = is_v ? l - LANES / 2 : l;   // eight-element chunk of the row
  int slot = -1, h = 0;
  long long row = 0;
  if (item < a.items) {
    row = a.items >> 31 ? item / a.d.Hkv : (long long)((unsigned)item / (unsigned)a.d.Hkv);   // (a division of 64 bits is a call)
    h = (int)(item - row * a.d.Hkv);
    slot = a.slot_map[row];
    if (slot >= (long long)a.d.n_pages * a.d.ps) slot = -1;
  }
  float x[8];
  const int exp = is_v ? a.v_exp : a.k_exp;
  unsigned most = 0u;   // largest magnitude, as an integer: what is not finite is larger than all that is
  if (slot >= 0) {
    load8(reinterpret_cast<const T*>(is_v ? a.v : a.k) + row * (is_v ? a.ldv : a.ldk) + (long long)h * Dh + 8 * c, x);
    const float f = __uint_as_float((unsigned)(127 - exp) << 23);   // 2^-exp
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= f;
      most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    }
  }
  // whether all of the row's head is finite: the ballot's bits of this group of lanes
  const unsigned group = LANES == 32 ? ~0u : 0xFFFFu << (threadIdx.x & 16);
  const bool fine = (__ballot_sync(~0u, most < 0x7F800000u) & group) == group;
  const float top = __uint_as_float(max(most, __shfl_xor_sync(~0u, most, 1)));
  if (slot < 0) return;
  // The quotient by IEEE division, rounded once more: a value half-way between two scales has few enough bits to be a quotient
  // that fp32 holds, and no other quotient rounds to it, so the result is the rounding of the exact quotient.
  unsigned short two;
  {
    const float t = __fdiv_rn(top, 7.f);
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(t));
  }
  unsigned byte = two & 0xFFu;
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)byte));
  float s = __half2float(__low2half(as_half2(r)));
  uint32_t word = 0u;   // codes without their offset of 8: four bits of the number
  if (!fine) byte = SCALE_NAN;
  else if (s > 0.f) {
    const float inv = __frcp_rn(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = nearest_code(x[i], s, inv);
      const int at = 4 * (i / 2 + 4 * (i % 2));
      word |= (__float_as_uint(t) << at) & (0xFu << at);
      x[i] = t - WHOLE;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
  }
  word ^= 0x88888888u;
  const int page = (unsigned)slot / (unsigned)a.d.ps, in = slot - page * a.d.ps, tau = in % CACHE_BLOCK;
  unsigned char* blk = a.pool + block_offset(a.d, page, in / CACHE_BLOCK, h);
  const int g = c >> 1;
  if (is_v) {
    *reinterpret_cast<uint32_t*>(blk + off_vc(Dh) + (tau >> 3) * (4 * Dh) + g * 64 + (tau & 7) * 8 + (c & 1) * 4) = word;
    if (!(c & 1)) blk[off_vs(Dh) + (tau >> 3) * (Dh / 2) + g * 8 + (tau & 7)] = (unsigned char)byte;
  } else {
    *reinterpret_cast<uint32_t*>(blk + tau * (Dh / 2) + c * 4) = word;
    if (!(c & 1)) blk[off_ks(Dh) + tau * (Dh / CACHE_GROUP) + g] = (unsigned char)byte;
  }
  void* val = is_v ? a.v_val : a.k_val;
  if (val) {
    const float f = fine ? s * __uint_as_float((unsigned)(127 + exp) << 23) : __int_as_float(0x7FC00000);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fine ? x[i] * f : f;   // exact: eight significant bits
    store8(reinterpret_cast<T*>(val) + (row * a.d.Hkv + h) * Dh + 8 * c, x);
  }
}

// ------------------------------------------------------------------------------------------------
// Commit.  A warp per (request, layer, head) holds the bytes of all moved rows before it writes one: sources and targets of
// a path overlap.  The CTAs of a request form a cluster, whose barrier lets the new length overwrite the old.  Bound by latency
// (nodes, table, bytes, then the writes): paths of up to eight rows of 32 requests, 12 layers of 8 heads, 6.4 us on the device
// for 4 MB; of one request with 36 layers 5.8 us for 0.6 MB.
// ------------------------------------------------------------------------------------------------
constexpr int COM_THREADS = 1024;   // at most: a warp for each layer and head of a request
// CTAs of a request: eight, and sixteen where a warp would have to take more than one layer and head (one request with 36 layers of
// 8 heads: 10.9 and 5.7 us, with 12 layers 5.2 and 5.0) and the device has clusters of sixteen.
constexpr int COM_CLUSTER = 8, COM_LARGE = 16;

struct CommitArgs {
  CacheDims d;
  int B, D, N, layers, cluster;
  size_t layer_stride;
  unsigned char* pool;
  const int *table, *seq_len, *status, *acc_len, *acc_node;   // status may be NULL
  int* seq_len_out;
};

template <int Dh>
__global__ void __launch_bounds__(COM_THREADS, 1) commit_kernel(const CommitArgs a) {
  constexpr int G = Dh / CACHE_GROUP;
  __shared__ long long from[DMAX], to[DMAX];   // byte offsets of the rows' blocks in layer 0, head 0; -1: no move
  __shared__ int ft[DMAX], tt[DMAX];           // tokens within the blocks
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x / a.cluster, part = blockIdx.x - b * a.cluster;
  const int lane = threadIdx.x & 31;
  const int seq = a.seq_len[b];
  const bool idle = seq < 0 || (a.status && a.status[b] != TS_OK);   // (no rows of this round: one that was refused pages wrote none)
  const int n = idle ? 0 : min(max(a.acc_len[b], 0), a.D);
  if (threadIdx.x < DMAX) {
    const int i = threadIdx.x;
    long long f = -1, t = -1;
    if (i < n) {
      const int node = a.acc_node[(size_t)b * a.D + i];
      const unsigned ps = a.d.ps, room = (unsigned)a.d.cols * ps, src = (unsigned)seq + 1u + (unsigned)node, dst = (unsigned)seq + 1u + (unsigned)i;   // (below 2^31 + 257)
      if (node >= 0 && node < a.N && src != dst && src < room && dst < room) {
        const int* row = a.table + (size_t)b * a.d.cols;
        const unsigned cs = src / ps, ct = dst / ps;
        f = block_offset(a.d, row[cs], (src - cs * ps) / CACHE_BLOCK, 0);
        t = block_offset(a.d, row[ct], (dst - ct * ps) / CACHE_BLOCK, 0);
        if (f < 0 || t < 0) f = t = -1;
      }
      ft[i] = src % CACHE_BLOCK; tt[i] = dst % CACHE_BLOCK;   // (pages are whole blocks)
    }
    from[i] = f; to[i] = t;
  }
  __syncthreads();
  // a lane's word of a token: K codes, then V codes; its byte: K scales, then V scales
  constexpr int W = Dh / 8;   // words of K codes (as many of V)
  const int warps = a.cluster * (blockDim.x / 32);
  for (int item = part * (blockDim.x / 32) + (threadIdx.x >> 5); item < a.layers * a.d.Hkv; item += warps) {
    const int layer = item / a.d.Hkv, h = item - layer * a.d.Hkv;
    unsigned char* base = a.pool + (size_t)layer * a.layer_stride + (size_t)h * (a.d.ps / CACHE_BLOCK) * cache_block_bytes(Dh);
    uint32_t word[DMAX];
    uint32_t byte[DMAX / 4];   // (packed: 1,024 threads have 64 registers each)
#pragma unroll
    for (int i = 0; i < DMAX / 4; ++i) byte[i] = 0u;
    const int j = lane % W;
    const bool has_word = lane < 2 * W, has_byte = lane < 2 * G;
    auto word_at = [&](unsigned char* blk, int tau) {
      return reinterpret_cast<uint32_t*>(lane < W ? blk + tau * (Dh / 2) + j * 4 : blk + off_vc(Dh) + (tau >> 3) * (4 * Dh) + (j >> 1) * 64 + (tau & 7) * 8 + (j & 1) * 4);
    };
    auto byte_at = [&](unsigned char* blk, int tau) {
      return lane < G ? blk + off_ks(Dh) + tau * G + lane : blk + off_vs(Dh) + (tau >> 3) * (8 * G) + (lane - G) * 8 + (tau & 7);
    };
#pragma unroll
    for (int i = 0; i < DMAX; ++i)
      if (i < n && from[i] >= 0) {
        if (has_word) word[i] = *word_at(base + from[i], ft[i]);
        if (has_byte) byte[i / 4] |= (uint32_t)*byte_at(base + from[i], ft[i]) << (8 * (i % 4));
      }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < DMAX; ++i)
      if (i < n && from[i] >= 0) {
        if (has_word) *word_at(base + to[i], tt[i]) = word[i];
        if (has_byte) *byte_at(base + to[i], tt[i]) = (unsigned char)(byte[i / 4] >> (8 * (i % 4)));
      }
    __syncwarp();
  }
  cooperative_groups::this_cluster().sync();   // all CTAs of the request have read its length
  if (part == 0 && threadIdx.x == 0) a.seq_len_out[b] = idle ? seq : seq + 1 + n;
}

// Clusters of sixteen CTAs are more than every device has to have: a partition of one may have none.
cudaError_t cache_setup(ts_ctx* ctx) {
  ctx->large_clusters = true;
  for (void (*kernel)(const CommitArgs) : {commit_kernel<128>, commit_kernel<64>}) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(COM_LARGE); cfg.blockDim = dim3(COM_THREADS);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = COM_LARGE; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    int fit = 0;
    e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (fit < 1) ctx->large_clusters = false;
  }
  return cudaSuccess;
}

}  // namespace ts

using namespace ts;

extern "C" size_t ts_cache_bytes(const ts_cache_layout* lay) {
  if (cache_layout_error(lay)) return 0;
  return (size_t)lay->n_pages * cache_dims(lay).page_bytes();
}

extern "C" int32_t ts_cache_reserve(ts_ctx* ctx, const ts_cache_layout* lay, int32_t B, const int32_t* seq_len, const int32_t* n_nodes,
                                    const int32_t* held, int32_t* free_pages, const int32_t* free_count, int32_t* block_table,
                                    int32_t* held_out, int32_t* free_count_out, int32_t* slot_map, int32_t* status, void* stream) {
  if (!ctx) return set_error(TS_ERR_INVALID, "ts_cache_reserve: null context");
  if (cache_layout_error(lay)) return set_layout_error("ts_cache_reserve", lay);
  const void* req[] = {seq_len, held, free_pages, free_count, block_table, held_out, free_count_out, slot_map, status};
  for (const void* p : req)
    if (bad_ptr4(p)) return set_error(TS_ERR_INVALID, "ts_cache_reserve: null or misaligned pointer");
  if (n_nodes && ((uintptr_t)n_nodes & 3u)) return set_error(TS_ERR_INVALID, "ts_cache_reserve: misaligned pointer");
  if (B < 1 || B > ctx->cfg.max_batch) return set_error(TS_ERR_INVALID, "ts_cache_reserve: B out of range");
  if (!on_ctx_device(ctx)) return set_error(TS_ERR_INVALID, "ts_cache_reserve: the context's device is not the current one");
  ReserveArgs a{};
  a.d = cache_dims(lay);
  a.B = B; a.rcap = n_nodes ? ctx->cfg.Nmax + 1 : 1;
  a.seq_len = seq_len; a.n_nodes = n_nodes; a.held = held; a.free_pages = free_pages; a.free_count = free_count; a.table = block_table;
  a.held_out = held_out; a.free_count_out = free_count_out; a.slot_map = slot_map; a.status = status;
  cudaError_t e = launch_reserve(ctx, a, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? TS_OK : set_cuda_error("ts_cache_reserve", e);
}

extern "C" int32_t ts_cache_append(ts_ctx* ctx, const ts_cache_layout* lay, int32_t rows, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                   const int32_t* slot_map, void* pool, void* k_val, void* v_val, void* stream) {
  if (!ctx) return set_error(TS_ERR_INVALID, "ts_cache_append: null context");
  if (cache_layout_error(lay)) return set_layout_error("ts_cache_append", lay);
  if (rows < 0) return set_error(TS_ERR_INVALID, "ts_cache_append: rows out of range");
  if (rows == 0) return TS_OK;
  const void* req[] = {k, v, pool};
  for (const void* p : req)
    if (bad_ptr(p)) return set_error(TS_ERR_INVALID, "ts_cache_append: null or misaligned pointer");
  if (bad_ptr4(slot_map)) return set_error(TS_ERR_INVALID, "ts_cache_append: null or misaligned pointer");
  if ((k_val && ((uintptr_t)k_val & 15u)) || (v_val && ((uintptr_t)v_val & 15u))) return set_error(TS_ERR_INVALID, "ts_cache_append: misaligned pointer");
  const int unit = lay->dtype == TS_DTYPE_BF16 ? 8 : 4;   // elements of 16 bytes
  const int64_t least = (int64_t)lay->Hkv * lay->Dh;
  if (ldk < least || ldv < least || ldk % unit || ldv % unit) return set_error(TS_ERR_INVALID, "ts_cache_append: row strides must cover Hkv * Dh elements and be multiples of 16 bytes");
  if (!on_ctx_device(ctx)) return set_error(TS_ERR_INVALID, "ts_cache_append: the context's device is not the current one");
  AppendArgs a{};
  a.d = cache_dims(lay);
  a.items = (long long)rows * lay->Hkv;
  a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv; a.slot_map = slot_map; a.pool = (unsigned char*)pool; a.k_val = k_val; a.v_val = v_val;
  a.k_exp = lay->k_exp; a.v_exp = lay->v_exp;
  const long long blocks = (a.items * (lay->Dh / 4) + APP_THREADS - 1) / APP_THREADS;
  if (blocks > 0x7FFFFFFFll) return set_error(TS_ERR_INVALID, "ts_cache_append: rows out of range");
  cudaStream_t st = (cudaStream_t)stream;
  void (*kernel)(const AppendArgs) = lay->dtype == TS_DTYPE_BF16 ? (lay->Dh == 128 ? append_kernel<__nv_bfloat16, 128> : append_kernel<__nv_bfloat16, 64>)
                                                                 : (lay->Dh == 128 ? append_kernel<float, 128> : append_kernel<float, 64>);
  cudaError_t e;
  {
    ProfScope ps(ctx, K_APPEND, st);
    e = launch_kernel(kernel, dim3((unsigned)blocks), dim3(APP_THREADS), 0, st, true, a);
  }
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? TS_OK : set_cuda_error("ts_cache_append", e);
}

static int32_t commit_paths(const char* call, ts_ctx* ctx, const ts_cache_layout* lay, int32_t B, int32_t layers, size_t layer_stride, void* pool,
                            const int32_t* block_table, const int32_t* seq_len, const int32_t* status, const int32_t* acc_len, const int32_t* acc_node,
                            int32_t* seq_len_out, void* stream) {
  auto refuse = [call](const char* why) {
    char msg[160];
    snprintf(msg, sizeof(msg), "%s: %s", call, why);
    return set_error(TS_ERR_INVALID, msg);
  };
  if (!ctx) return refuse("null context");
  if (cache_layout_error(lay)) return set_layout_error(call, lay);
  if (bad_ptr(pool)) return refuse("null or misaligned pointer");
  const void* req[] = {block_table, seq_len, acc_len, acc_node, seq_len_out};
  for (const void* p : req)
    if (bad_ptr4(p)) return refuse("null or misaligned pointer");
  if (B < 1 || B > ctx->cfg.max_batch) return refuse("B out of range");
  if (layers < 1 || layers > 4096) return refuse("layers out of range");
  if (layers > 1 && (layer_stride < ts_cache_bytes(lay) || layer_stride % 16)) return refuse("layer stride must cover a layer's pool and be a multiple of 16 bytes");
  if (!on_ctx_device(ctx)) return refuse("the context's device is not the current one");
  CommitArgs a{};
  a.d = cache_dims(lay);
  a.B = B; a.D = ctx->cfg.D; a.N = ctx->cfg.Nmax; a.layers = layers; a.layer_stride = layer_stride; a.pool = (unsigned char*)pool;
  a.table = block_table; a.seq_len = seq_len; a.status = status; a.acc_len = acc_len; a.acc_node = acc_node; a.seq_len_out = seq_len_out;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  {
    ProfScope ps(ctx, K_COMMIT, st);
    cudaLaunchConfig_t cfg = {};
    const int items = layers * lay->Hkv;
    a.cluster = items > COM_CLUSTER * (COM_THREADS / 32) && ctx->large_clusters ? COM_LARGE : COM_CLUSTER;
    cfg.gridDim = dim3(B * a.cluster); cfg.blockDim = dim3(std::min(COM_THREADS, (items + a.cluster - 1) / a.cluster * 32)); cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization; attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, lay->Dh == 128 ? commit_kernel<128> : commit_kernel<64>, a);
  }
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? TS_OK : set_cuda_error(call, e);
}

extern "C" int32_t ts_cache_commit(ts_ctx* ctx, const ts_cache_layout* lay, int32_t B, int32_t layers, size_t layer_stride, void* pool,
                                   const int32_t* block_table, const int32_t* seq_len, const int32_t* acc_len, const int32_t* acc_node,
                                   int32_t* seq_len_out, void* stream) {
  return commit_paths("ts_cache_commit", ctx, lay, B, layers, layer_stride, pool, block_table, seq_len, nullptr, acc_len, acc_node, seq_len_out, stream);
}

extern "C" int32_t ts_cache_commit_granted(ts_ctx* ctx, const ts_cache_layout* lay, int32_t B, int32_t layers, size_t layer_stride, void* pool,
                                           const int32_t* block_table, const int32_t* seq_len, const int32_t* status, const int32_t* acc_len,
                                           const int32_t* acc_node, int32_t* seq_len_out, void* stream) {
  if (bad_ptr4(status)) return set_error(TS_ERR_INVALID, "ts_cache_commit_granted: null or misaligned pointer");
  return commit_paths("ts_cache_commit_granted", ctx, lay, B, layers, layer_stride, pool, block_table, seq_len, status, acc_len, acc_node, seq_len_out, stream);
}

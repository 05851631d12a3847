// Attention of a round's rows over the 4-bit cache: the entry point, the kernel for few query rows a kv head, and the kernel
// that joins the pieces of cut units.
#include "ts_attn.cuh"
#include "ts_tc.cuh"

namespace ts {

// ------------------------------------------------------------------------------------------------
// Few rows: 8 NT query rows of one kv head a unit, on mma.sync with the cache's tokens on the rows of the matrix
// instruction (S^T = K Q^T, O^T = V^T P^T), so that one instruction of 16 x 8 serves eight query rows (four query heads a kv head
// leave half of its columns empty; with rows on the other side three quarters would be).  Single tokens of 64 requests of 1,000 to 16,000 tokens with eight kv heads of 128 channels (626 MB of
// cache): 169 us, 3.7 TB/s.  The copies alone take 107 to 119 us; what is left are the fixed latencies of unpacking 4,096 codes a block of 16
// tokens, which three warps a scheduler do not cover: 329 instructions a block, issued in 48 % of the slots.
// ------------------------------------------------------------------------------------------------
constexpr int FEW_WARPS = 4;
constexpr int FEW_THREADS = FEW_WARPS * 32;
// Blocks a warp takes in a step: what a step costs besides them is shared, and their chains run side by side.  (2, 3, 4 blocks: the
// batch above takes 206, 184, 198 us; with four the registers leave room for two CTAs an SM.)
constexpr int FEW_BLOCKS = 3;
constexpr int FEW_TOKENS = FEW_BLOCKS * CACHE_BLOCK;
// A lead of eight steps (64 requests of 1,000 to 16,000 tokens, us, with leads of 0, 2, 4, 8, 12, 16: 184, 185, 179, 170, 173, 176).
template <int NT> using FewShape = AttnShape<8 * NT, FEW_TOKENS, 8>;

template <int Dh, int NT>
struct FewPlan {
  static constexpr int QT = 8 * NT;
  static constexpr int BLK = cache_block_bytes(Dh);
  static constexpr int STEP = FEW_BLOCKS * BLK;
  static constexpr int STAGES = 2;
  static constexpr int ROW = Dh + 4;                       // floats between rows of the merge buffer
  static constexpr int RING = FEW_WARPS * STAGES * STEP;
  static constexpr int MERGE = FEW_WARPS * QT * (ROW + 2) * 4;
  static constexpr int SMEM = RING + MERGE;
};

// A block to shared memory by the warp's lanes, 16 bytes each at a time.  (Bulk copies take as long, and barriers besides.)
template <int BLK>
__device__ __forceinline__ void copy_block(uint32_t dst, const unsigned char* src, int lane) {
#pragma unroll
  for (int k = 0; k < BLK; k += 512)
    if (k + 512 <= BLK || k + lane * 16 < BLK) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + k + lane * 16), "l"(src + k + lane * 16) : "memory");
}
__device__ __forceinline__ void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the first product of a sum
__device__ __forceinline__ void mma_16816_first(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// The query rows of a unit as B operands: lane (g, t) holds channels t Dh/4 .. of row g of each tile of eight.  A row is
// multiplied by the power of two that brings its largest element to 2^14..2^15: bf16 then is exact in fp16 down to 2^-38 of
// that element.  fp32 is split into two fp16 parts, exact to 2^-22.  The scale's sign goes to the queries, its magnitude to f: what
// a column's sums are multiplied with (not 0, so that a masked sum, -inf, has weight 0 whatever the scale is).
template <int Dh, int NT, bool F32>
struct Queries {
  static constexpr int REGS = Dh / 8;   // registers a tile
  uint32_t hi[NT][REGS];
  uint32_t lo[F32 ? NT : 1][F32 ? REGS : 1];
  float f[NT][2];

  __device__ __forceinline__ void load(const AttnArgs& a, const AttnUnit& u, int h, int first, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int idx = first + 8 * n + g;
      float x[Dh / 4];
      if (idx < u.rows * a.d.G) {
        const size_t at = head_row(a, u.b, h, idx, a.ldq) + t * (Dh / 4);
        if (F32) {
          const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + at);
#pragma unroll
          for (int i = 0; i < Dh / 16; ++i) {
            const float4 v = __ldg(p + i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
          }
        } else {
          const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + at);
#pragma unroll
          for (int i = 0; i < Dh / 32; ++i) unpack_bf16x8(__ldg(p + i), x + 8 * i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < Dh / 4; ++i) x[i] = 0.f;
      }
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < Dh / 4; ++i) top = fmaxf(top, fabsf(x[i]));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
      const int e = max((int)(__float_as_uint(top) >> 23), 20);         // biased exponent; 2^(141 - e) has to be a float
      // (a row with an infinity has no finite score: it becomes NaN, so that one whose scores are all -inf is no empty row)
      const float up = e < 255 ? copysignf(__uint_as_float((unsigned)(127 + 141 - e) << 23), a.qk) : NAN;
      const float mine = fmaxf(1e-30f, fabsf(a.qk) * __uint_as_float((unsigned)(127 + e - 141) << 23));
#pragma unroll
      for (int i = 0; i < REGS; ++i) {
        const float x0 = x[2 * i] * up, x1 = x[2 * i + 1] * up;
        const __half2 v = __floats2half2_rn(x0, x1);
        hi[n][i] = as_u32(v);
        if (F32) lo[n][i] = as_u32(__floats2half2_rn(x0 - __low2float(v), x1 - __high2float(v)));
      }
      f[n][0] = __shfl_sync(~0u, mine, 8 * t);
      f[n][1] = __shfl_sync(~0u, mine, 8 * t + 4);
    }
  }
};

// Scores of a block's 16 tokens, before the factors of the columns: rows g, g + 8 (tokens), columns 2t, 2t + 1 (queries).
template <int Dh, int NT, bool F32>
__device__ __forceinline__ void score_block(const unsigned char* blk, const Queries<Dh, NT, F32>& q, float (&s)[NT][4], int g, int t) {
  constexpr int KW = Dh / 32;        // words of a token's K codes that a lane holds
  uint32_t kw[2][KW];
  __half2 sc[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const unsigned char* row = blk + (g + 8 * e) * (Dh / 2) + t * (Dh / 8);
    if (Dh == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(row);
      kw[e][0] = v.x; kw[e][1] = v.y; kw[e][KW - 2] = v.z; kw[e][KW - 1] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(row);
      kw[e][0] = v.x; kw[e][1] = v.y;
    }
    const unsigned char* sp = blk + off_ks(Dh) + (g + 8 * e) * (Dh / CACHE_GROUP) + t * (Dh / 64);
    sc[e] = k_scales(Dh == 128 ? *reinterpret_cast<const unsigned short*>(sp) : *sp);
  }
#pragma unroll
  for (int i = 0; i < KW; ++i) {
    uint32_t x[2][4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const __half2 ss = Dh == 128 && i >= KW / 2 ? __high2half2(sc[e]) : __low2half2(sc[e]);
      unpack8(kw[e][i], ss, __hmul2(ss, __float2half2_rn(-1032.f)), __hmul2(ss, __float2half2_rn(-72.f)), x[e]);
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const uint32_t fr[4] = {x[0][2 * v], x[1][2 * v], x[0][2 * v + 1], x[1][2 * v + 1]};
      const int r = 4 * i + 2 * v;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (F32) {
          // each step's sum apart and added in fp32: the instruction's own accumulation rounds towards zero
          float c[4];
          mma_16816_first(c, fr, q.lo[F32 ? n : 0][F32 ? r : 0], q.lo[F32 ? n : 0][F32 ? r + 1 : 0]);
          mma_16816(c, fr, q.hi[n][r], q.hi[n][r + 1]);
#pragma unroll
          for (int k = 0; k < 4; ++k) s[n][k] = r == 0 ? c[k] : s[n][k] + c[k];
        } else if (r == 0) mma_16816_first(s[n], fr, q.hi[n][r], q.hi[n][r + 1]);
        else mma_16816(s[n], fr, q.hi[n][r], q.hi[n][r + 1]);
      }
    }
  }
}

// O^T += V^T P^T for a block: lane (g, t) holds Dh/8 channels of tokens 2t, 2t + 1 of both octets.
template <int Dh, int NT, bool F32>
__device__ __forceinline__ void value_block(const unsigned char* blk, const uint32_t (&ph)[NT][2], const uint32_t (&pl)[F32 ? NT : 1][2], float (&o)[NT][Dh / 16][4], int g, int t) {
  constexpr int VW = Dh / 64;   // words of a token that a lane holds
  uint32_t va[2][VW], vb[2][VW];
  __half2 vs[2], c1032[2], c72[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const unsigned char* oct = blk + off_vc(Dh) + e * (4 * Dh);
    if (Dh == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(oct + g * 64 + t * 16);
      va[e][0] = v.x; va[e][VW - 1] = v.y; vb[e][0] = v.z; vb[e][VW - 1] = v.w;
    } else {
      va[e][0] = *reinterpret_cast<const uint32_t*>(oct + (g >> 1) * 64 + t * 16 + (g & 1) * 4);
      vb[e][0] = *reinterpret_cast<const uint32_t*>(oct + (g >> 1) * 64 + t * 16 + 8 + (g & 1) * 4);
    }
    vs[e] = v_scales(*reinterpret_cast<const unsigned short*>(blk + off_vs(Dh) + e * (Dh / 2) + (Dh == 128 ? g : g >> 1) * 8 + 2 * t));
    c1032[e] = __hmul2(vs[e], __float2half2_rn(-1032.f));
    c72[e] = __hmul2(vs[e], __float2half2_rn(-72.f));
  }
#pragma unroll
  for (int i = 0; i < VW; ++i) {
    uint32_t lo[2][4], hi[2][4];   // even and odd channels of the word, tokens in the halves
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      unpack8(__byte_perm(va[e][i], vb[e][i], 0x5410), vs[e], c1032[e], c72[e], lo[e]);
      unpack8(__byte_perm(va[e][i], vb[e][i], 0x7632), vs[e], c1032[e], c72[e], hi[e]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t fr[4] = {lo[0][j], hi[0][j], lo[1][j], hi[1][j]};
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float* acc = o[n][4 * i + j];
        if (F32) {
          float c[4];
          mma_16816_first(c, fr, pl[F32 ? n : 0][0], pl[F32 ? n : 0][1]);
          mma_16816(c, fr, ph[n][0], ph[n][1]);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[k] += c[k];
        } else {
          mma_16816(acc, fr, ph[n][0], ph[n][1]);
        }
      }
    }
  }
}

template <int Dh, int NT, bool F32>
__global__ void __launch_bounds__(FEW_THREADS, F32 || NT > 1 ? 2 : 3) attn_few_kernel(const AttnArgs a) {
  using P = FewPlan<Dh, NT>;
  using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
  constexpr int QT = P::QT, ST = P::STAGES, BLK = P::BLK;
  constexpr int MT = Dh / 16;        // tiles of 16 channels
  constexpr float ROOM = F32 ? 0.f : 8.f, LIFT = F32 ? 15.f : 7.f;
  extern __shared__ __align__(128) unsigned char smem[];
  float* merge = reinterpret_cast<float*>(smem + P::RING);
  float* merge_ml = merge + FEW_WARPS * QT * P::ROW;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  pdl_wait();
  pdl_launch_dependents();
  AttnUnit u;
  int first_step;
  long long steps_;
  if (!attn_locate<FewShape<NT>, FEW_THREADS>(a, u, first_step, steps_)) return;
  const int steps = (int)steps_;

  // The copies run ahead of the arithmetic, across units (each warp has a ring and copy groups of its own): the warp's steps are
  // w, w + 4, .. of the CTA's.  The cursor stands at step fj of unit fu, in column fc and block fin of that page; the table's
  // entries are read a step ahead.
  unsigned char* ring = smem + w * ST * P::STEP;
  const int per = a.d.ps / CACHE_BLOCK, adv = FEW_WARPS * FEW_BLOCKS, adv_c = adv / per, adv_in = adv - adv_c * per;
  AttnUnit fu = u;
  int fj = first_step + w, fleft = steps - w, fc = fj * FEW_BLOCKS / per, fin = fj * FEW_BLOCKS - fc * per, fh = fu.v / fu.nq;
  int fslot = 0, page = -1, inner = 0;   // (the first lanes: a block each)
  uint32_t present = 0;                  // four bits a slot: its blocks that have a page
  auto look_up = [&]() {
    if (fleft <= 0) return;
    if (fj >= fu.n) {
      do {
        fj -= fu.n;
        next_unit<FewShape<NT>>(a, fu);
      } while (fj >= fu.n);
      fc = fj * FEW_BLOCKS / per; fin = fj * FEW_BLOCKS - fc * per; fh = fu.v / fu.nq;
    }
    inner = fin + lane;
    int c = fc;
    while (inner >= per) { inner -= per; ++c; }
    const unsigned last = (unsigned)fu.seq + (unsigned)fu.rows - 1u;   // the request's last token; a block behind it is not fetched
    page = lane < FEW_BLOCKS && c < a.d.cols && (unsigned)(fj * FEW_BLOCKS + lane) * CACHE_BLOCK <= last ? __ldg(a.table + (size_t)fu.b * a.d.cols + c) : -1;
  };
  auto fetch = [&]() {
    if (fleft > 0) {
      const long long off = block_offset(a.d, page, inner, fh);
      const unsigned there = __ballot_sync(~0u, off >= 0);
      present = (present & ~(0xFu << (4 * fslot))) | there << (4 * fslot);
      const uint32_t dst = smem_u32(ring + fslot * P::STEP);
#pragma unroll
      for (int k = 0; k < FEW_BLOCKS; ++k) {
        const long long at = __shfl_sync(~0u, off, k);
        if (at >= 0) copy_block<BLK>(dst + k * BLK, a.pool + at, lane);
      }
      if (++fslot == ST) fslot = 0;
      fj += FEW_WARPS; fleft -= FEW_WARPS;
      fc += adv_c; fin += adv_in;
      if (fin >= per) { fin -= per; ++fc; }
      look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look_up();
#pragma unroll
  for (int s = 0; s < ST; ++s) fetch();

  int slot = 0;
  int mine = w;                                   // the warp's next step, counted from the CTA's first
  int pos = 0;                                    // the segment's first
  while (pos < steps) {
    const int h = u.v / u.nq, first = (u.v - h * u.nq) * QT;
    const int j0 = pos == 0 ? first_step : 0;     // step of the unit at which the segment begins
    const int seg = min(u.n - j0, steps - pos);
    Queries<Dh, NT, F32> q;
    q.load(a, u, h, first, lane);
    float o[NT][MT][4], m[NT][2], ref[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][i][c] = 0.f;
      m[n][0] = m[n][1] = -INFINITY; ref[n][0] = ref[n][1] = 0.f; l[n][0] = l[n][1] = 0.f;
    }
    for (; mine < pos + seg; mine += FEW_WARPS) {
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
      __syncwarp();
      const int here = present >> (4 * slot) & 0xFu;
      const unsigned char* blk = ring + slot * P::STEP;
      float s[FEW_BLOCKS][NT][4];
#pragma unroll
      for (int k = 0; k < FEW_BLOCKS; ++k) score_block<Dh, NT, F32>(blk + k * BLK, q, s[k], g, t);
      // ---- weights
      const int tok0 = (j0 + mine - pos) * FEW_TOKENS;
      const bool masked = tok0 > u.seq - FEW_TOKENS || here != (1 << FEW_BLOCKS) - 1;
      uint32_t ph[FEW_BLOCKS][NT][2], pl[FEW_BLOCKS][F32 ? NT : 1][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (masked) {
#pragma unroll
          for (int k = 0; k < FEW_BLOCKS; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int rel = tok0 + k * CACHE_BLOCK + g + 8 * (c >> 1) - u.seq, idx = first + 8 * n + 2 * t + (c & 1);
              const bool sees = ((here >> k) & 1) && (rel < 0 || row_sees(a, u.b, tree_row(a, idx), rel, u.rows));
              if (!sees) s[k][n][c] = -INFINITY;
            }
        }
        // The reference of the exponents moves only when a score passes it by more than ROOM: weights stay below
        // 2^(ROOM + LIFT) = 2^15, and LIFT keeps small ones out of fp16's subnormals.
        float top[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[c] = fmaxf(s[0][n][c], s[0][n][c + 2]);
#pragma unroll
          for (int k = 1; k < FEW_BLOCKS; ++k) top[c] = fmaxf(top[c], fmaxf(s[k][n][c], s[k][n][c + 2]));
          top[c] *= q.f[n][c];
        }
        if (__any_sync(~0u, top[0] > m[n][0] || top[1] > m[n][1])) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) top[c] = fmaxf(top[c], __shfl_xor_sync(~0u, top[c], x));
            if (top[c] > m[n][c]) {
              const float r = m[n][c] == -INFINITY ? 0.f : ex2(ref[n][c] - (top[c] - LIFT));
              m[n][c] = top[c] + ROOM; ref[n][c] = top[c] - LIFT;
              l[n][c] *= r;
#pragma unroll
              for (int i = 0; i < MT; ++i) { o[n][i][c] *= r; o[n][i][c + 2] *= r; }
            }
          }
        }
#pragma unroll
        for (int k = 0; k < FEW_BLOCKS; ++k) {
          float e[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) e[c] = ex2(fmaf(s[k][n][c], q.f[n][c & 1], -ref[n][c & 1]));
          l[n][0] += e[0] + e[2]; l[n][1] += e[1] + e[3];
          const __half2 h0 = __floats2half2_rn(e[0], e[1]), h1 = __floats2half2_rn(e[2], e[3]);
          ph[k][n][0] = transpose8(as_u32(h0)); ph[k][n][1] = transpose8(as_u32(h1));
          if (F32) {
            pl[k][F32 ? n : 0][0] = transpose8(as_u32(__floats2half2_rn(e[0] - __low2float(h0), e[1] - __high2float(h0))));
            pl[k][F32 ? n : 0][1] = transpose8(as_u32(__floats2half2_rn(e[2] - __low2float(h1), e[3] - __high2float(h1))));
          }
        }
      }
#pragma unroll
      for (int k = 0; k < FEW_BLOCKS; ++k) value_block<Dh, NT, F32>(blk + k * BLK, ph[k], pl[k], o, g, t);
      __syncwarp();   // every lane has read the slot that the next copies go to
      if (++slot == ST) slot = 0;
      fetch();
    }
    // ---- the four warps' parts of the unit
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[n][c];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(~0u, sum, x);
        const int row = w * QT + 8 * n + 2 * t + c;
        if (g == 0) { merge_ml[2 * row] = m[n][c] == -INFINITY ? -INFINITY : ref[n][c]; merge_ml[2 * row + 1] = sum; }
#pragma unroll
        for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(merge + row * P::ROW + g * (Dh / 8) + 2 * i) = make_float2(o[n][i][c], o[n][i][c + 2]);
      }
    __syncthreads();
    const bool whole = seg == u.n;
    const size_t piece = ((size_t)blockIdx.x * 2 + (j0 > 0 ? 0 : 1)) * QT;
    for (int e = threadIdx.x; e < QT * Dh; e += FEW_THREADS) {
      const int row = e / Dh, ch = e - row * Dh, idx = first + row;
      if (idx >= u.rows * a.d.G) continue;
      float top = -INFINITY, wm[FEW_WARPS], sum = 0.f, x = 0.f;
#pragma unroll
      for (int k = 0; k < FEW_WARPS; ++k) top = fmaxf(top, wm[k] = merge_ml[2 * (k * QT + row)]);
#pragma unroll
      for (int k = 0; k < FEW_WARPS; ++k) {
        const float r = part_weight(wm[k], top);
        sum += r * merge_ml[2 * (k * QT + row) + 1];
        x += r * merge[(k * QT + row) * P::ROW + ch];
      }
      if (whole) {
        store_out(reinterpret_cast<T*>(a.out) + out_row(a, u.b, h, idx) + ch, x * row_inv(sum) * a.vo);
        if (ch == 0 && a.lse) a.lse[lse_row(a, u.b, h, idx)] = row_lse(top, sum);
      } else {
        a.part[(piece + row) * Dh + ch] = x;
        if (ch == 0) { a.part_ml[2 * (piece + row)] = top; a.part_ml[2 * (piece + row) + 1] = sum; }
      }
    }
    __syncthreads();
    pos += seg;
    if (pos < steps) next_unit<FewShape<NT>>(a, u);
  }
}

// ------------------------------------------------------------------------------------------------
// Join: a CTA takes some rows of a cut unit, a warp a row; where there are many pieces, all its warps one row after the
// other.  The pieces are added in an order that depends on their number only.  Bound by latency (the record, then sums and
// pieces, which are loaded together): 1.6 us of 9.8 for one request of 517 tokens, 6 of 47 for two contexts of up to
// 131,000 (fp32), 6 of 96 for 32 trees, 14 of 235 for 8 requests with trees of 120 to 256 nodes (up to 38 MB of pieces, from L2).
// ------------------------------------------------------------------------------------------------
constexpr int JOIN_WARPS = 8;
// Rows a CTA: few rows are cut into many pieces, which a CTA's warps share (1, 2, 4, 8 rows: the request 12.1, 10.3, 10.0, 10.0 us, two
// contexts of 130,000 tokens 58, 57, 58, 61, four of up to 3,000 13.9, 13.2, 14.9, 14.9); of many rows fewer mean more CTAs
// that find nothing (8, 16, 32 rows: the 32 trees 117, 114, 116 us).
constexpr int JOIN_FEW = 2, JOIN_MANY = 16;
constexpr int JOIN_BATCH = 4;   // pieces whose loads a warp has in flight (8: the trees 121 us for 117)

template <int Dh, typename T>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attn_join_kernel(const AttnArgs a, int QT, int per) {
  constexpr int V = Dh / 32;   // channels of a lane
  using Vec = typename std::conditional<V == 4, float4, float2>::type;
  __shared__ float acc[JOIN_WARPS][Dh], red[JOIN_WARPS];
  pdl_wait();
  pdl_launch_dependents();
  const AttnRecord r = a.records[blockIdx.x];
  if (r.first < 0) return;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, n = r.last - r.first + 1;
  const int h = r.v / r.nq, first = (r.v - h * r.nq) * QT, r0 = blockIdx.y * per;
  const int rows = min(min(QT, r0 + per), r.rows * a.d.G - first);        // of the tile, that are there
  const int rw = n > 2 * JOIN_WARPS ? JOIN_WARPS : 1, part = rw > 1 ? w : 0;   // warps a row
  for (int row = r0 + (rw > 1 ? 0 : w); row < rows; row += rw > 1 ? 1 : JOIN_WARPS) {
    // piece k: the first begins at or before the unit and is its CTA's last; the others begin within it
    auto at = [&](int k) { return ((size_t)(r.first + k) * 2 + (k == 0 ? 1 : 0)) * QT + row; };
    float2 ml[JOIN_BATCH];
    Vec y[JOIN_BATCH];
    auto load = [&](int k0) {
#pragma unroll
      for (int i = 0; i < JOIN_BATCH; ++i) {
        const int k = k0 + i * rw;
        ml[i] = make_float2(-INFINITY, 0.f);
        y[i] = Vec{};
        if (k < n) {
          ml[i] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at(k));
          y[i] = *reinterpret_cast<const Vec*>(a.part + at(k) * Dh + lane * V);
        }
      }
    };
    load(part);   // (on their way together with what the largest reference needs)
    float top = -INFINITY;
    for (int k = lane; k < n; k += 32) top = fmaxf(top, a.part_ml[2 * at(k)]);
#pragma unroll
    for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
    float sum = 0.f, x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = 0.f;
    for (int k0 = part; k0 < n;) {
#pragma unroll
      for (int i = 0; i < JOIN_BATCH; ++i) {
        const float wgt = part_weight(ml[i].x, top);
        sum += wgt * ml[i].y;
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] += wgt * reinterpret_cast<const float*>(&y[i])[v];
      }
      k0 += JOIN_BATCH * rw;
      if (k0 < n) load(k0);
    }
    if (rw > 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) acc[w][lane * V + v] = x[v];
      if (lane == 0) red[w] = sum;
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = 0.f;
#pragma unroll
      for (int k = 0; k < JOIN_WARPS; ++k) {
        sum += red[k];
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] += acc[k][lane * V + v];
      }
      __syncthreads();
      if (w > 0) continue;
    }
    const int idx = first + row;
    T* out = reinterpret_cast<T*>(a.out) + out_row(a, r.b, h, idx) + lane * V;
    const float inv = row_inv(sum) * a.vo;
#pragma unroll
    for (int v = 0; v < V; ++v) store_out(out + v, x[v] * inv);
    if (lane == 0 && a.lse) a.lse[lse_row(a, r.b, h, idx)] = row_lse(top, sum);
  }
}

cudaError_t attn_join(ts_ctx* ctx, const AttnArgs& a, int QT, bool f32, cudaStream_t st) {
  ProfScope ps(ctx, K_ATTN_JOIN, st);
  const int per = QT > 16 ? JOIN_MANY : JOIN_FEW;
  void (*kernel)(const AttnArgs, int, int) = f32 ? (a.d.Dh == 128 ? attn_join_kernel<128, float> : attn_join_kernel<64, float>)
                                            : (a.d.Dh == 128 ? attn_join_kernel<128, __nv_bfloat16> : attn_join_kernel<64, __nv_bfloat16>);
  return launch_kernel(kernel, dim3(a.grid, (QT + per - 1) / per), dim3(JOIN_WARPS * 32), 0, st, true, a, QT, per);
}

static size_t round256(size_t n) { return (n + 255) / 256 * 256; }

size_t attn_workspace(int grid, int QT, int Dh) {
  return round256((size_t)grid * sizeof(AttnRecord)) + round256((size_t)grid * 2 * QT * Dh * 4) + round256((size_t)grid * 2 * QT * 2 * 4);
}

void attn_place(AttnArgs& a, int QT, char* ws) {
  a.records = (AttnRecord*)ws;
  a.part = (float*)(ws + round256((size_t)a.grid * sizeof(AttnRecord)));
  a.part_ml = (float*)((char*)a.part + round256((size_t)a.grid * 2 * QT * a.d.Dh * 4));
}

// Query rows of a unit and CTAs of a launch.  Two tiles of eight rows share the unpacked keys and values, one tile leaves room for
// three CTAs an SM (32 requests of 500 to 8,000 tokens, one tile and two: 9 rows 94 and 77 us, 16 rows 97 and 85; 8 rows need
// only one; fp32 with 64 channels, 32 rows behind two contexts of up to 131,000 tokens 57 and 47).  fp32 with 128 channels takes
// one: queries and weights of two parts each do not fit twice without spilling (16 requests of up to 4,000 tokens 26 and 30 us).
static int few_tiles_of(const CacheDims& d, int rcap, bool f32) { return (long long)rcap * d.G > 8 && !(f32 && d.Dh == 128) ? 2 : 1; }
static int few_ctas(int nt, bool f32) { return f32 || nt > 1 ? 2 : 3; }

static size_t attn_few_workspace(const ts_ctx* ctx, const CacheDims& d, bool f32) {
  size_t most = 0;
  for (int nt = 1; nt <= 2; ++nt) {
    const size_t n = attn_workspace(ctx->num_sms * few_ctas(nt, f32), 8 * nt, d.Dh);
    most = n > most ? n : most;
  }
  return most;
}

template <int Dh, int NT, bool F32>
static cudaError_t launch_few(ts_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  using P = FewPlan<Dh, NT>;
  cudaError_t e;
  {
    ProfScope ps(ctx, K_ATTN_FEW, st);
    e = launch_kernel(attn_few_kernel<Dh, NT, F32>, dim3(a.grid), dim3(FEW_THREADS), P::SMEM, st, true, a);
  }
  return e != cudaSuccess ? e : attn_join(ctx, a, P::QT, F32, st);
}

cudaError_t attn_setup(ts_ctx* ctx) {
  cudaError_t e = cudaSuccess;
  auto allow = [&](auto kernel) { if (e == cudaSuccess) e = allow_all_smem(kernel, ctx->max_smem); };
  allow(attn_few_kernel<128, 1, false>); allow(attn_few_kernel<128, 2, false>); allow(attn_few_kernel<128, 1, true>);
  allow(attn_few_kernel<64, 1, false>); allow(attn_few_kernel<64, 2, false>); allow(attn_few_kernel<64, 1, true>); allow(attn_few_kernel<64, 2, true>);
  if (e == cudaSuccess) e = attn_many_setup(ctx);
  // the same split of L1 and shared memory as the kernels before it and after: an SM that changes it has to run empty first
  auto shared = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared); };
  shared(attn_join_kernel<128, float>); shared(attn_join_kernel<64, float>); shared(attn_join_kernel<128, __nv_bfloat16>); shared(attn_join_kernel<64, __nv_bfloat16>);
  return e;
}

static cudaError_t attn_few_launch(ts_ctx* ctx, AttnArgs a, bool f32, char* ws, cudaStream_t st) {
  const int nt = few_tiles_of(a.d, a.rcap, f32);
  a.grid = ctx->num_sms * few_ctas(nt, f32);
  a.min_steps = FEW_WARPS;
  attn_place(a, 8 * nt, ws);
  const auto launch = a.d.Dh == 128 ? f32 ? launch_few<128, 1, true> : nt == 2 ? launch_few<128, 2, false> : launch_few<128, 1, false>
                                    : f32 ? nt == 2 ? launch_few<64, 2, true> : launch_few<64, 1, true> : nt == 2 ? launch_few<64, 2, false> : launch_few<64, 1, false>;
  return launch(ctx, a, st);
}

// Which kernel: tiles of 16 rows read the keys and values again for every tile, tiles of 128 pay for rows that are not there (32
// requests of 500 to 8,000 tokens, few and many: 16 rows 85 and 114 us, 17 rows 144 and 115, 32 rows 157 and 116).
static bool takes_many(const CacheDims& d, int rcap, bool f32) { return !f32 && (long long)rcap * d.G > 16; }

}  // namespace ts

using namespace ts;

extern "C" size_t ts_tree_attention_workspace_bytes(const ts_ctx* ctx, const ts_cache_layout* lay, int32_t B) {
  if (!ctx || cache_layout_error(lay) || B < 1 || B > ctx->cfg.max_batch) return 0;
  const CacheDims d = cache_dims(lay);
  const size_t few = attn_few_workspace(ctx, d, lay->dtype == TS_DTYPE_F32), many = attn_many_workspace(ctx, d);
  return lay->dtype == TS_DTYPE_F32 || few > many ? few : many;
}

extern "C" int32_t ts_tree_attention(ts_ctx* ctx, const ts_cache_layout* lay, int32_t B, const void* q, int64_t ldq, const void* pool,
                                     const int32_t* block_table, const int32_t* seq_len, const int32_t* n_nodes, const uint64_t* mask,
                                     float scale, void* out, int64_t ldo, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx) return set_error(TS_ERR_INVALID, "ts_tree_attention: null context");
  if (cache_layout_error(lay)) return set_layout_error("ts_tree_attention", lay);
  const void* req[] = {q, pool, out, ws};
  for (const void* p : req)
    if (bad_ptr(p)) return set_error(TS_ERR_INVALID, "ts_tree_attention: null or misaligned pointer");
  if (bad_ptr4(block_table) || bad_ptr4(seq_len) || (n_nodes && bad_ptr4(n_nodes)) || (lse && bad_ptr4(lse)) || ((uintptr_t)mask & 7u))
    return set_error(TS_ERR_INVALID, "ts_tree_attention: null or misaligned pointer");
  if (mask && !n_nodes) return set_error(TS_ERR_INVALID, "ts_tree_attention: a mask needs n_nodes");
  if (B < 1 || B > ctx->cfg.max_batch) return set_error(TS_ERR_INVALID, "ts_tree_attention: B out of range");
  const bool f32 = lay->dtype == TS_DTYPE_F32;
  const int64_t unit = f32 ? 4 : 8, least = (int64_t)lay->Hq * lay->Dh;
  if (ldq < least || ldo < least || ldq % unit || ldo % unit) return set_error(TS_ERR_INVALID, "ts_tree_attention: row strides must cover Hq * Dh elements and be multiples of 16 bytes");
  if (!(fabsf(scale) <= 1e30f && fabsf(ldexpf(scale, lay->k_exp)) <= 1e30f)) return set_error(TS_ERR_INVALID, "ts_tree_attention: scale (and scale * 2^k_exp) must be at most 1e30 in magnitude");
  if (ws_bytes < ts_tree_attention_workspace_bytes(ctx, lay, B)) return set_error(TS_ERR_WORKSPACE, "ts_tree_attention: workspace too small");
  if (!on_ctx_device(ctx)) return set_error(TS_ERR_INVALID, "ts_tree_attention: the context's device is not the current one");
  AttnArgs a{};
  a.d = cache_dims(lay);
  a.B = B; a.rcap = n_nodes ? ctx->cfg.Nmax + 1 : 1; a.N = ctx->cfg.Nmax; a.words = (ctx->cfg.Nmax + 63) / 64;
  a.q = q; a.ldq = ldq; a.pool = (const unsigned char*)pool; a.table = block_table; a.seq_len = seq_len; a.n_nodes = n_nodes; a.mask = mask;
  a.by_g = (unsigned)(((1ull << 32) + a.d.G - 1) / a.d.G);   // (G = 1: not used)
  a.qk = ldexpf(scale * LOG2E, K_SHIFT + lay->k_exp); a.vo = ldexpf(1.f, V_SHIFT + lay->v_exp);
  a.out = out; a.ldo = ldo; a.lse = lse; a.limit = ctx->wait_limit; a.lost = ctx->test_mode & TS_TEST_LOST_ARRIVAL ? 16u : 0u;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = takes_many(a.d, a.rcap, f32) ? attn_many_launch(ctx, a, (char*)ws, st) : attn_few_launch(ctx, a, f32, (char*)ws, st);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? TS_OK : set_cuda_error("ts_tree_attention", e);
}

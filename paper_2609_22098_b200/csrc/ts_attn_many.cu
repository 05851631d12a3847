// Attention over the 4-bit cache for many query rows a kv head (trees, chunks of prompts) on the 5th-generation tensor cores.
//
// One CTA an SM with a piece of the line of steps (128 tokens of one head).  Roles:
//   loader        one warp: bulk copies of the cache's blocks into a ring of 64 tokens a stage
//   converters    eight warps: codes to fp16 (exact) in the operands' swizzled layout, K and V two stages each
//   issuer        one warp: S = Q K^T (128 rows x 128 tokens) and O += P V, accumulators and P in tensor memory
//   softmax       two groups of four warps, a thread a query row: scores to weights in place, fp16
// A unit has up to 256 query rows.  With more than 128 the groups take a tile of 128 rows each, and both read the same
// converted keys and values; with fewer they take the same rows and every other step, and their halves are joined at the end.
// Either way one group's exponentials run beside the other's matrix products.
#include "ts_attn.cuh"
#include "ts_tc.cuh"

namespace ts {

constexpr int MANY_TOKENS = 128;                  // a step
constexpr int MANY_QT = 256;
constexpr int MANY_SOFT = 8, MANY_CONV = 8;       // warps
constexpr int MANY_ISSUE = MANY_SOFT + MANY_CONV, MANY_LOAD = MANY_ISSUE + 1, MANY_WARPS = MANY_LOAD + 1;
constexpr int MANY_THREADS = MANY_WARPS * 32;
constexpr int MANY_RAW = 3;                       // stages of raw blocks
constexpr int MANY_RAW_BLOCKS = 4;                // blocks of a stage: 64 tokens
constexpr int MANY_PRESENT = 16;                  // steps whose missing blocks are remembered; the loader is at most six ahead

template <int Dh>
struct ManyPlan {
  static constexpr int TILE = 128 * Dh * 2;       // bytes of 128 rows of fp16
  static constexpr int SLAB = 128 * 128;          // 128 rows of 64 channels
  static constexpr int RAW = MANY_RAW_BLOCKS * cache_block_bytes(Dh);
  static constexpr int Q = 0, K = 2 * TILE, V = 4 * TILE, R = 6 * TILE;
  static constexpr int SMEM = 6 * TILE + MANY_RAW * RAW + 1024;   // (the dynamic array is aligned to 1,024 in the kernel)
  static constexpr uint32_t O = 256;              // tensor memory columns: S of the groups at 0 and 128, P in their first 64
};

struct ManyBars {
  uint64_t raw_full[MANY_RAW], raw_free[MANY_RAW];
  uint64_t k_full[2], k_free[2], v_full[2], v_free[2];
  uint64_t q_full, s_full[2], p_full[2], o_full[2];
};

// D = f32, A = B = f16, M = 128, N = n; B MN-major (values) or K-major (keys)
__device__ __forceinline__ uint32_t many_idesc(int n, bool mn_major) { return (1u << 4) | (mn_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24); }
__device__ __forceinline__ void mma_tmem_a(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
#define TS_R4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];"
      : TS_R4(r, 0), TS_R4(r, 4), TS_R4(r, 8), TS_R4(r, 12), TS_R4(r, 16), TS_R4(r, 20), TS_R4(r, 24), TS_R4(r, 28)
      : "r"(taddr) : "memory");
}
#undef TS_R4
#define TS_W4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::TS_W4(r, 0), TS_W4(r, 4), TS_W4(r, 8), TS_W4(r, 12), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, "
      "%29, %30, %31};"
      ::TS_W4(r, 0), TS_W4(r, 4), TS_W4(r, 8), TS_W4(r, 12), TS_W4(r, 16), TS_W4(r, 20), TS_W4(r, 24), TS_W4(r, 28), "r"(taddr) : "memory");
}
#undef TS_W4
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

struct ManyShared {
  ManyBars bars;
  uint32_t tmem;
  int abort;
  unsigned char present[MANY_PRESENT];   // a bit for each block of a step
  float ml[2][128][2];                   // reference and sum of the two groups, where they share rows
};

// The steps of a CTA's piece that belong to one unit.
struct ManySegment { int h, first, j0, n, two; bool whole; };
template <int Dh>
__device__ __forceinline__ ManySegment many_segment(const AttnArgs& a, const AttnUnit& u, long long start, long long end, long long at) {
  ManySegment s;
  s.h = u.v / u.nq;
  s.first = (u.v - s.h * u.nq) * MANY_QT;
  s.j0 = (int)(at - u.t0);
  s.n = (int)min((long long)(u.n - s.j0), end - at);
  s.two = u.rows * a.d.G - s.first > 128;
  s.whole = s.n == u.n;
  return s;
}

// ---- loader -------------------------------------------------------------------------------------------------------------
template <int Dh>
__device__ void many_load(const AttnArgs& a, ManyShared& sh, unsigned char* raw, AttnUnit u, long long start, long long end) {
  using P = ManyPlan<Dh>;
  const int lane = threadIdx.x & 31, per = a.d.ps / CACHE_BLOCK, half_steps = (int)(end - start) * 2;
  long long at = start;
  int page = -1, inner = 0, h = u.v / u.nq;
  // entry of the table for this lane's block of half-step `hs`
  auto look_up = [&](int hs) {
    if (hs >= half_steps) return;
    const long long p = start + (hs >> 1);
    while (p >= u.t0 + u.n) { next_unit<MANY_QT, MANY_TOKENS>(a, u); h = u.v / u.nq; }
    const int jb = (int)(p - u.t0) * (MANY_TOKENS / CACHE_BLOCK) + (hs & 1) * MANY_RAW_BLOCKS + lane, c = jb / per;
    inner = jb - c * per;
    const unsigned last = (unsigned)u.seq + (unsigned)u.rows - 1u;
    page = lane < MANY_RAW_BLOCKS && c < a.d.cols && (unsigned)jb * CACHE_BLOCK <= last ? __ldg(a.table + (size_t)u.b * a.d.cols + c) : -1;
  };
  look_up(0);
  int slot = 0;
  uint32_t phase = 0, seen = 0;
  for (int hs = 0; hs < half_steps; ++hs) {
    const long long off = block_offset(a.d, page, inner, h);
    const unsigned there = __ballot_sync(~0u, off >= 0);
    look_up(hs + 1);
    if (hs >= MANY_RAW && !__all_sync(~0u, mbar_wait(&sh.bars.raw_free[slot], phase ^ 1u, (volatile int*)&sh.abort, nullptr, a.limit))) break;
    if (lane == 0) {
      unsigned char* pr = &sh.present[(hs >> 1) % MANY_PRESENT];
      *pr = (unsigned char)((hs & 1) ? *pr | there << 4 : there);
      mbar_expect_tx(&sh.bars.raw_full[slot], __popc(there) * cache_block_bytes(Dh));
    }
    __syncwarp();
    if (off >= 0)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   ::"r"(smem_u32(raw + slot * P::RAW + lane * cache_block_bytes(Dh))), "l"(a.pool + off), "r"((uint32_t)cache_block_bytes(Dh)), "r"(smem_u32(&sh.bars.raw_full[slot])) : "memory");
    __syncwarp();
    seen |= 1u << slot;
    if (++slot == MANY_RAW) { slot = 0; phase ^= 1u; }
  }
  // after a wait that gave up copies may still be on their way: (the last use of a slot completes the phase before the next)
  if (sh.abort)
    for (int s = 0; s < MANY_RAW; ++s)
      if (seen >> s & 1u)
        for (uint32_t i = 0; i < a.limit && !mbar_try_wait(&sh.bars.raw_full[s], s < slot ? phase : phase ^ 1u); ++i) __nanosleep(100);
}

// ---- converters ---------------------------------------------------------------------------------------------------------
// K [token][channel], K-major: rows of 64 channels (128 bytes), 16-byte chunks exchanged by the row's last three bits.
template <int Dh>
__device__ __forceinline__ void convert_keys(const unsigned char* raw, unsigned char* dst, int half, int tid) {
  // a thread: 64 bytes of results, Dh/8 bytes of a token's codes (Dh = 128: 32 channels; 64: 16)
  const int tok = tid >> 2, q = tid & 3, row = half * 64 + tok;
  const unsigned char* blk = raw + (tok >> 4) * cache_block_bytes(Dh);
  const unsigned char* sp = blk + off_ks(Dh) + (tok & 15) * (Dh / CACHE_GROUP) + q * (Dh / 64);
  constexpr int W = Dh / 32;
  uint32_t w[W];
  __half2 sc;
  int turn = 0;
  if (Dh == 128) {
    const uint4 v = *reinterpret_cast<const uint4*>(blk + (tok & 15) * (Dh / 2) + q * 16);
    sc = k_scales(*reinterpret_cast<const unsigned short*>(sp));
    // lanes of the two halves of a row write to other banks: the second pair of words first
    turn = q & 2;
    w[0] = turn ? v.z : v.x; w[1] = turn ? v.w : v.y; w[W - 2] = turn ? v.x : v.z; w[W - 1] = turn ? v.y : v.w;
    if (turn) sc = __lowhigh2highlow(sc);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(blk + (tok & 15) * (Dh / 2) + q * 8);
    w[0] = v.x; w[1] = v.y;
    sc = k_scales(*sp);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const __half2 ss = Dh == 128 && i >= W / 2 ? __high2half2(sc) : __low2half2(sc);
    uint32_t x[4];
    unpack8(w[i], ss, __hmul2(ss, __float2half2_rn(-1032.f)), __hmul2(ss, __float2half2_rn(-72.f)), x);
    const int chunk = q * W + (i ^ turn);   // of eight channels
    *reinterpret_cast<uint4*>(dst + (chunk >> 3) * ManyPlan<Dh>::SLAB + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
  }
}
// V [token][channel], MN-major: the same rows; tokens are the contraction.
template <int Dh>
__device__ __forceinline__ void convert_values(const unsigned char* raw, unsigned char* dst, int half, int tid) {
#pragma unroll
  for (int k = 0; k < Dh / 64; ++k) {
    const int item = tid + k * (MANY_CONV * 32);               // [block][octet][group][token]
    const int t8 = item & 7, rest = item >> 3, g = rest % (Dh / CACHE_GROUP), oct = rest / (Dh / CACHE_GROUP), row = half * 64 + oct * 8 + t8;
    const unsigned char* blk = raw + (oct >> 1) * cache_block_bytes(Dh);
    const uint2 w = *reinterpret_cast<const uint2*>(blk + off_vc(Dh) + (oct & 1) * (4 * Dh) + g * 64 + t8 * 8);
    const uint32_t byte = blk[off_vs(Dh) + (oct & 1) * (Dh / 2) + g * 8 + t8];
    const __half2 ss = v_scales(byte * 0x101u), c1032 = __hmul2(ss, __float2half2_rn(-1032.f)), c72 = __hmul2(ss, __float2half2_rn(-72.f));
    unsigned char* out = dst + (g >> 2) * ManyPlan<Dh>::SLAB + row * 128;
    uint32_t x[4];
    unpack8(w.x, ss, c1032, c72, x);
    *reinterpret_cast<uint4*>(out + ((((g & 3) * 2) ^ (row & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
    unpack8(w.y, ss, c1032, c72, x);
    *reinterpret_cast<uint4*>(out + ((((g & 3) * 2 + 1) ^ (row & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
  }
}
template <int Dh>
__device__ void many_convert(const AttnArgs& a, ManyShared& sh, unsigned char* smem, int steps) {
  using P = ManyPlan<Dh>;
  const int tid = threadIdx.x - MANY_SOFT * 32, lane = threadIdx.x & 31;
  volatile int* abort = (volatile int*)&sh.abort;
  int slot = 0;
  uint32_t phase = 0;
  for (int j = 0; j < steps; ++j) {
    const int st = j & 1;
    const uint32_t par = ((uint32_t)(j >> 1) & 1u) ^ 1u;   // of the use before
    unsigned char *k = smem + P::K + st * P::TILE, *v = smem + P::V + st * P::TILE;
    int s2 = slot;
    uint32_t p2 = phase;
    if (j >= 2 && !mbar_wait(&sh.bars.k_free[st], par, abort, nullptr, a.limit)) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!mbar_wait(&sh.bars.raw_full[s2], p2, abort, nullptr, a.limit)) return;
      convert_keys<Dh>(smem + P::R + s2 * P::RAW, k, half, tid);
      if (++s2 == MANY_RAW) { s2 = 0; p2 ^= 1u; }
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.bars.k_full[st]);
    if (j >= 2 && !mbar_wait(&sh.bars.v_free[st], par, abort, nullptr, a.limit)) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      convert_values<Dh>(smem + P::R + slot * P::RAW, v, half, tid);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.bars.raw_free[slot]);
      if (++slot == MANY_RAW) { slot = 0; phase ^= 1u; }
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.bars.v_full[st]);
  }
}

// ---- issuer -------------------------------------------------------------------------------------------------------------
template <int Dh>
__device__ void many_issue(const AttnArgs& a, ManyShared& sh, unsigned char* smem, AttnUnit u, long long start, long long end) {
  using P = ManyPlan<Dh>;
  volatile int* abort = (volatile int*)&sh.abort;
  const uint32_t tmem = sh.tmem, id_s = many_idesc(MANY_TOKENS, false), id_o = many_idesc(Dh, true);
  const uint64_t qd = smem_desc(smem_u32(smem + P::Q), 16u, 1024u), kd = smem_desc(smem_u32(smem + P::K), 16u, 1024u), vd = smem_desc(smem_u32(smem + P::V), P::SLAB, 1024u);
  uint32_t p_count[2] = {0u, 0u};   // weights waited for, per group
  int base = 0, segments = 0;       // steps before this segment
  auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait(bar, parity, abort, nullptr, a.limit)); };
  for (long long at = start; at < end;) {
    const ManySegment s = many_segment<Dh>(a, u, start, end, at);
    const int ops = s.two ? 2 * s.n : s.n;
    if (!wait(&sh.bars.q_full, segments & 1)) return;
    // product i: group i & 1, step i / 2 (two tiles) or i; its P V is issued two products later
    for (int i = 0; i < ops + 2; ++i) {
      const int tile = i & 1;
      if (i >= 2) {
        const int j = s.two ? (i - 2) >> 1 : i - 2, gj = base + j;
        if (!wait(&sh.bars.p_full[tile], p_count[tile] & 1u)) return;
        ++p_count[tile];
        if (!wait(&sh.bars.v_full[gj & 1], (gj >> 1) & 1)) return;
        tc_fence_after();
        if (elect_one()) {
          const uint32_t d = tmem + P::O + tile * Dh, pa = tmem + tile * 128;
          const uint64_t b = vd + (uint64_t)((gj & 1) * (P::TILE >> 4));
          const uint32_t fresh = i < 4 ? 0u : 1u;   // the group's first of the unit
#pragma unroll
          for (int ks = 0; ks < MANY_TOKENS / 16; ++ks) mma_tmem_a(d, pa + ks * 8, b + (uint64_t)(ks * 128), id_o, ks > 0 ? 1u : fresh);
          mma_commit(&sh.bars.o_full[tile]);
          if (!s.two || tile == 1) mma_commit(&sh.bars.v_free[gj & 1]);
        }
        __syncwarp();
      }
      if (i < ops) {
        const int j = s.two ? i >> 1 : i, gj = base + j;
        if (!wait(&sh.bars.k_full[gj & 1], (gj >> 1) & 1)) return;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t qa = qd + (uint64_t)((s.two ? tile : 0) * (P::TILE >> 4)), b = kd + (uint64_t)((gj & 1) * (P::TILE >> 4));
#pragma unroll
          for (int ks = 0; ks < Dh / 16; ++ks) {
            const uint64_t off = (uint64_t)((ks >> 2) * (P::SLAB >> 4) + (ks & 3) * 2);
            mma_bf16(tmem + tile * 128, qa + off, b + off, id_s, ks > 0 ? 1u : 0u);
          }
          mma_commit(&sh.bars.s_full[tile]);
          if (!s.two || tile == 1) mma_commit(&sh.bars.k_free[gj & 1]);
        }
        __syncwarp();
      }
    }
    base += s.n;
    ++segments;
    at += s.n;
    if (at < end) next_unit<MANY_QT, MANY_TOKENS>(a, u);
  }
}

// ---- softmax ------------------------------------------------------------------------------------------------------------
// Bit c: whether tree row i sees the token at place rel0 + c behind the prefix (rel0 + c < 0: in it).
__device__ __forceinline__ uint32_t sees32(const AttnArgs& a, int b, int i, int rel0, int rows) {
  if (rel0 + 31 < 0) return ~0u;
  if (i >= rows || rel0 >= rows) return rel0 < 0 && i < rows ? (1u << -rel0) - 1u : 0u;
  auto low = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };   // the first n bits
  uint32_t bits = low(rows - rel0) & (a.mask ? ~0u : low(i + 1 - rel0));
  if (a.mask) {
    // bits 0.. of the row: the anchor, then the nodes' bits
    const uint64_t* row = a.mask + ((size_t)b * a.N + (i - 1)) * a.words;
    uint32_t on = low(-rel0) | (rel0 <= 0 ? 1u << -rel0 : 0u);   // the prefix and the anchor (rel0 > -32 here)
    if (i > 0) {
      const int first = rel0 - 1;   // bit of the mask that stands at place 0; may be negative
      uint64_t word = 0;
      if (first < 0) word = row[0] << -first;
      else {
        word = row[first >> 6] >> (first & 63);
        if ((first & 63) && (first >> 6) + 1 < a.words) word |= row[(first >> 6) + 1] << (64 - (first & 63));
      }
      on |= (uint32_t)word;
    }
    bits &= on;
  }
  return bits;
}

// The row's queries as fp16 in the operand's layout, times a power of two (see Queries in ts_attn.cu); returns the factor that
// makes its scores exponents of two.  chunks c0 .. c1 - 1 (of eight channels) are written.
template <int Dh>
__device__ __forceinline__ float load_query(const AttnArgs& a, const AttnUnit& u, int h, int idx, unsigned char* dst, int row, int c0, int c1) {
  uint4 v[Dh / 8];
  const bool used = idx < u.rows * a.d.G;
  const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)u.b * a.rcap + idx / a.d.G) * a.ldq + (size_t)(h * a.d.G + idx % a.d.G) * Dh;
  uint32_t top = 0;   // largest magnitude, as bf16 bits in both halves (magnitudes compare as integers)
#pragma unroll
  for (int c = 0; c < Dh / 8; ++c) {
    v[c] = used ? __ldg(reinterpret_cast<const uint4*>(src) + c) : make_uint4(0u, 0u, 0u, 0u);
    top = __vmaxu2(top, __vmaxu2(__vmaxu2(v[c].x & 0x7FFF7FFFu, v[c].y & 0x7FFF7FFFu), __vmaxu2(v[c].z & 0x7FFF7FFFu, v[c].w & 0x7FFF7FFFu)));
  }
  const uint32_t big = max(top & 0xFFFFu, top >> 16);
  const int e = max((int)(big >> 7), 20);
  // (the sign of the scale goes to the queries: the largest score is the factor times the largest sum)
  const float up = copysignf(__uint_as_float((unsigned)(127 + 141 - e) << 23), a.qk);
#pragma unroll
  for (int c = 0; c < Dh / 8; ++c) {
    if (c < c0 || c >= c1) continue;
    float x[8];
    unpack_bf16x8(v[c], x);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = as_u32(__floats2half2_rn(x[2 * i] * up, x[2 * i + 1] * up));
    *reinterpret_cast<uint4*>(dst + (c >> 3) * ManyPlan<Dh>::SLAB + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return fabsf(a.qk) * __uint_as_float((unsigned)(127 + e - 141) << 23);
}

template <int Dh>
__device__ void many_softmax(const AttnArgs& a, ManyShared& sh, unsigned char* smem, AttnUnit u, long long start, long long end) {
  using P = ManyPlan<Dh>;
  constexpr float ROOM = 8.f, LIFT = 7.f;
  volatile int* abort = (volatile int*)&sh.abort;
  const int grp = threadIdx.x >> 7, row = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t lanes = (uint32_t)(row & 96) << 16, ts = sh.tmem + lanes + grp * 128, to = sh.tmem + lanes + P::O;
  uint32_t count = 0;   // products of this group
  int base = 0;
  bool alive = true;
  for (long long at = start; at < end;) {
    const ManySegment s = many_segment<Dh>(a, u, start, end, at);
    const int idx = s.first + (s.two ? grp * 128 : 0) + row, i = idx / a.d.G;
    // both groups write half of a shared tile; their own where they have one
    const float f = load_query<Dh>(a, u, s.h, idx, smem + P::Q + (s.two ? grp * P::TILE : 0), row, s.two ? 0 : grp * (Dh / 16), s.two ? Dh / 8 : (grp + 1) * (Dh / 16));
    fence_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.bars.q_full);
    float m = -INFINITY, ref = 0.f, l = 0.f;
    int done = 0;   // products of this segment
    for (int j = s.two ? 0 : grp; j < s.n && alive; j += s.two ? 1 : 2) {
      alive = __all_sync(~0u, mbar_wait(&sh.bars.s_full[grp], count & 1u, abort, nullptr, a.limit));
      if (!alive) break;
      tc_fence_after();
      const int tok0 = (s.j0 + j) * MANY_TOKENS;
      const unsigned here = sh.present[(base + j) % MANY_PRESENT];
      const bool masked = tok0 > u.seq - MANY_TOKENS || here != 0xFFu;
      auto seen = [&](int c) {   // tokens of chunk c that the row sees
        const unsigned two = here >> (2 * c);
        return ((two & 1u ? 0xFFFFu : 0u) | (two & 2u ? 0xFFFF0000u : 0u)) & sees32(a, u.b, i, tok0 + 32 * c - u.seq, u.rows);
      };
      float top = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t r[32];
        tmem_ld32(ts + 32 * c, r);
        tmem_ld_wait();
        if (masked) {
          const uint32_t on = seen(c);
#pragma unroll
          for (int k = 0; k < 32; ++k) r[k] = on >> k & 1u ? r[k] : 0xFF800000u;
        }
#pragma unroll
        for (int k = 0; k < 32; k += 2) top = fmaxf(top, fmaxf(__uint_as_float(r[k]), __uint_as_float(r[k + 1])));
      }
      top = top == -INFINITY ? top : top * f;
      if (__any_sync(~0u, top > m)) {
        // (weights of at most 2^15; the reference moves when a score passes it by more than ROOM)
        const bool up = top > m;
        const float r = m == -INFINITY ? 0.f : ex2(ref - (top - LIFT));
        if (up) { ref = top - LIFT; l *= r; }
        if (__any_sync(~0u, up && m != -INFINITY)) {
          // the products before have to be in the sum that is scaled
          alive = __all_sync(~0u, mbar_wait(&sh.bars.o_full[grp], (count - 1u) & 1u, abort, nullptr, a.limit));
          if (!alive) break;
          tc_fence_after();
          const float k = up ? r : 1.f;
#pragma unroll
          for (int c = 0; c < Dh / 32; ++c) {
            uint32_t x[32];
            tmem_ld32(to + grp * Dh + 32 * c, x);
            tmem_ld_wait();
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] = __float_as_uint(__uint_as_float(x[q]) * k);
            tmem_st32(to + grp * Dh + 32 * c, x);
          }
          tmem_st_wait();
        }
        if (up) m = top + ROOM;
      }
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t r[32], w[16];
        tmem_ld32(ts + 32 * c, r);
        tmem_ld_wait();
        const uint32_t on = masked ? seen(c) : ~0u;
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          float e0 = ex2(fmaf(__uint_as_float(r[k]), f, -ref)), e1 = ex2(fmaf(__uint_as_float(r[k + 1]), f, -ref));
          if (masked) { e0 = on >> k & 1u ? e0 : 0.f; e1 = on >> (k + 1) & 1u ? e1 : 0.f; }
          l0 += e0; l1 += e1;
          w[k / 2] = as_u32(__floats2half2_rn(e0, e1));
        }
        tmem_st16(ts + 16 * c, w);
      }
      l += l0 + l1;
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.bars.p_full[grp]);
      ++count;
      ++done;
    }
    // ---- results: a group's own tile, or half of the channels of the rows that both share
    if (alive && done > 0) alive = __all_sync(~0u, mbar_wait(&sh.bars.o_full[grp], (count - 1u) & 1u, abort, nullptr, a.limit));
    float sum = l, top = m == -INFINITY ? m : ref, w0 = 1.f, w1 = 0.f;   // weights of the groups' parts
    bool other = false;
    if (!s.two) {
      sh.ml[grp][row][0] = top; sh.ml[grp][row][1] = l;
      soft_sync();            // (both groups' products are complete: each has waited for its own)
      const float t0 = sh.ml[0][row][0], t1 = sh.ml[1][row][0], l0 = sh.ml[0][row][1], l1 = sh.ml[1][row][1];
      top = fmaxf(t0, t1);
      w0 = part_weight(t0, top); w1 = part_weight(t1, top);
      sum = w0 * l0 + w1 * l1;
      other = s.n > 1;        // else the second group's sum was never written
    }
    if (!alive || *abort) sum = NAN;
    tc_fence_after();
    const bool used = idx < u.rows * a.d.G;
    const size_t piece = ((size_t)blockIdx.x * 2 + (start > u.t0 ? 0 : 1)) * MANY_QT + (s.two ? grp * 128 : 0) + row;
    const float inv = s.whole ? row_inv(sum) * a.vo : 1.f;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out) + (used ? out_row(a, u.b, s.h, idx) : 0);
    const int c_lo = s.two ? 0 : grp * (Dh / 64), c_hi = s.two ? Dh / 32 : (grp + 1) * (Dh / 64);
    for (int c = c_lo; c < c_hi; ++c) {
      uint32_t x[32];
      tmem_ld32(to + (s.two ? grp * Dh : 0) + 32 * c, x);
      tmem_ld_wait();
      float v[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) v[k] = w0 * __uint_as_float(x[k]);
      if (other) {
        tmem_ld32(to + Dh + 32 * c, x);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] += w1 * __uint_as_float(x[k]);
      }
      if (used && s.whole) {
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
          uint32_t w[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const __nv_bfloat162 h2 = __floats2bfloat162_rn(v[k + 2 * q] * inv, v[k + 2 * q + 1] * inv);
            w[q] = *reinterpret_cast<const uint32_t*>(&h2);
          }
          *reinterpret_cast<uint4*>(out + 32 * c + k) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if (used) {
#pragma unroll
        for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(a.part + piece * Dh + 32 * c + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
      }
    }
    if (used && (s.two || grp == 0)) {
      if (!s.whole) { a.part_ml[2 * piece] = top; a.part_ml[2 * piece + 1] = sum; }
      else if (a.lse) a.lse[lse_row(a, u.b, s.h, idx)] = row_lse(top, sum);
    }
    tc_fence_before();
    if (!s.two) soft_sync();   // both have read both sums, before the next unit's products overwrite them
    base += s.n;
    at += s.n;
    if (at < end) next_unit<MANY_QT, MANY_TOKENS>(a, u);
  }
}

template <int Dh>
__global__ void __launch_bounds__(MANY_THREADS, 1) attn_many_kernel(const AttnArgs a) {
  using P = ManyPlan<Dh>;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ ManyShared sh;
  unsigned char* smem = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    ManyBars& b = sh.bars;
    sh.abort = 0;
    for (int s = 0; s < MANY_RAW; ++s) { mbar_init(&b.raw_full[s], 1); mbar_init(&b.raw_free[s], MANY_CONV); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&b.k_full[s], MANY_CONV); mbar_init(&b.k_free[s], 1);
      mbar_init(&b.v_full[s], MANY_CONV); mbar_init(&b.v_free[s], 1);
      mbar_init(&b.s_full[s], 1); mbar_init(&b.p_full[s], 4); mbar_init(&b.o_full[s], 1);
    }
    mbar_init(&b.q_full, MANY_SOFT);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  AttnUnit u;
  long long start, end;
  int active;
  if (!attn_locate<MANY_QT, MANY_TOKENS, MANY_THREADS>(a, u, start, end, active)) return;
  if (warp == MANY_ISSUE) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp < MANY_SOFT) many_softmax<Dh>(a, sh, smem, u, start, end);
  else if (warp < MANY_ISSUE) many_convert<Dh>(a, sh, smem, (int)(end - start));
  else if (warp == MANY_ISSUE) many_issue<Dh>(a, sh, smem, u, start, end);
  else many_load<Dh>(a, sh, smem + P::R, u, start, end);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MANY_ISSUE) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(512u) : "memory");
}

cudaError_t attn_many_setup(ts_ctx* ctx) {
  const cudaError_t e = allow_all_smem(attn_many_kernel<128>, ctx->max_smem);
  return e != cudaSuccess ? e : allow_all_smem(attn_many_kernel<64>, ctx->max_smem);
}

size_t attn_many_workspace(const ts_ctx* ctx, const CacheDims& d) { return attn_workspace(ctx->num_sms, MANY_QT, d.Dh); }

cudaError_t attn_many_launch(ts_ctx* ctx, AttnArgs a, char* ws, cudaStream_t st) {
  a.grid = ctx->num_sms;
  a.min_steps = 1;
  attn_place(a, MANY_QT, ws);
  cudaError_t e;
  {
    ProfScope ps(ctx, K_ATTN_MANY, st);
    e = a.d.Dh == 128 ? launch_kernel(attn_many_kernel<128>, dim3(a.grid), dim3(MANY_THREADS), ManyPlan<128>::SMEM, st, true, a)
                      : launch_kernel(attn_many_kernel<64>, dim3(a.grid), dim3(MANY_THREADS), ManyPlan<64>::SMEM, st, true, a);
  }
  return e != cudaSuccess ? e : attn_join(ctx, a, MANY_QT, false, st);
}

}  // namespace ts

// Attention over the 4-bit cache for many query rows a kv head (trees, chunks of prompts) on the 5th-generation tensor cores.
//
// One CTA an SM with a piece of the line of steps (128 tokens of one head).  Roles:
//   loader        one warp: bulk copies of the cache's blocks into a ring of 64 tokens a stage
//   converters    two warps for K, two for V: codes to fp16 (exact) in the operands' swizzled layout, two stages each
//   issuer        one thread: S = Q K^T (128 rows x 128 tokens) and O += P V, accumulators and P in tensor memory
//   softmax       two groups of eight warps, two threads a query row with 64 of a step's scores each: scores to weights in
//                 place, fp16.  (With one thread a row a step's scores took it 2,500 cycles, which its next product waited for.)
// A unit has up to 256 query rows.  With more than 128 the groups take a tile of 128 rows each, and both read the same
// converted keys and values; with fewer they take the same rows and every other step, and their halves are joined at the end.
// Either way one group's exponentials run beside the other's matrix products.
//
// Trees of 120 to 256 nodes of 8 requests behind 2,000 to 16,000 tokens, 32 query heads on 4 of 128 channels: 235 us on the device (join and
// all), 0.83 PFLOP/s, 51 % of what a large matrix product reaches.  Trees of 8 to 30 nodes of 32 requests behind 500 to 6,000 tokens, 8 kv heads: 96 us, 1.3 TB/s.
// What bounds it is the chain of a tile (scores, their largest, weights, product with V, then the next scores, which need the
// weights' columns) and the waits between its links, which two groups cover in part; with one tile the converters (64 KB of
// fp16 a step) are as busy.
#include <string.h>

#include "ts_attn.cuh"
#include "ts_tc.cuh"

namespace ts {

constexpr int MANY_TOKENS = 128;                  // a step
constexpr int MANY_QT = 256;
// A lead of four steps (trees of 32 requests behind 500 to 6,000 tokens and the crowded trees above, us, with leads of 2, 3, 4, 6: 105
// and 247, 100 and 242, 98 and 236, 101 and 236; without one the trees took a third longer).  Steps
// with one and with two tiles count alike: the former are shorter, but what they wait for is the same (counted as 2 to 3 they
// took the crowded trees 6 % longer).
using ManyShape = AttnShape<MANY_QT, MANY_TOKENS, 4>;
constexpr int MANY_SOFT = 16, MANY_CONV = 4;      // warps (converters: half for K, half for V)
constexpr int MANY_CT = MANY_CONV / 2 * 32;       // threads of either kind
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
  static constexpr uint32_t O = 256;              // tensor memory columns: S of the groups at 0 and 128; P of 64 tokens in the first 32 columns of their scores
};

struct ManyBars {
  uint64_t raw_full[MANY_RAW], raw_free[MANY_RAW];
  uint64_t k_full[2], v_full[2], k_free[2][2], v_free[2][2];   // (free: by group and stage)
  uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
  uint64_t issued;   // all products
};

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
// the wait, with the registers that it waits for: nothing that uses them can be moved before it
#define TS_B4(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3])
__device__ __forceinline__ void tmem_ld32_wait(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : TS_B4(r, 0), TS_B4(r, 4), TS_B4(r, 8), TS_B4(r, 12), TS_B4(r, 16), TS_B4(r, 20), TS_B4(r, 24), TS_B4(r, 28)::"memory");
}
__device__ __forceinline__ void tmem_ld16_wait(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : TS_B4(r, 0), TS_B4(r, 4), TS_B4(r, 8), TS_B4(r, 12)::"memory");
}
#undef TS_B4
#define TS_W4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::TS_W4(r, 0), TS_W4(r, 4), TS_W4(r, 8), TS_W4(r, 12), "r"(taddr) : "memory");
}
#undef TS_W4
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// all softmax warps; the two that share 32 rows
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(MANY_SOFT * 32) : "memory"); }
__device__ __forceinline__ void pair_sync(int quad) { asm volatile("bar.sync %0, 64;" ::"r"(2 + quad) : "memory"); }

// a CTA's piece: its first unit, the number of its first step there, its steps
struct ManyPiece { AttnUnit u; int steps, first; };

struct ManyShared {
  ManyPiece piece;
  ManyBars bars;
  uint32_t tmem;
  int abort;
  unsigned char present[MANY_PRESENT];   // a bit for each block of a step
  float f[2][128];                       // factors of the rows' scores, by tile
  float top[2][2][128];                  // by group and half: largest scores of a step; at a unit's end the rows' references
  float sum[2][2][128];                  // and sums
  AttnUnit unit[MANY_SOFT];              // what a softmax warp works on
};

// A copy from shared memory that is made where it stands.  Every role reads its own copy of the piece (kept in registers across the
// parting of the roles it was spilled in all of them), and the softmax warps read their unit again behind its steps.  Spilled
// words of 768 threads do not fit beside so much shared memory in L1: 220 bytes a thread made trees 14 % slower.
template <class T>
__device__ __forceinline__ T copy_of(const T& in) {
  T out;
  constexpr int W = sizeof(T) / 4;
  static_assert(sizeof(T) % 4 == 0, "words");
  uint32_t w[W];
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const volatile uint32_t*>(&in)[i];
  memcpy(&out, w, sizeof(out));
  return out;
}

// The steps of a CTA's piece that belong to one unit: n from j0 on; `left` steps of the piece are to be taken.
struct ManySegment { int h, first, j0, n, two; bool whole; };
__device__ __forceinline__ int many_first(const AttnUnit& u) { return u.v % u.nq * MANY_QT; }
__device__ __forceinline__ ManySegment many_segment(const AttnArgs& a, const AttnUnit& u, int j0, int left) {
  ManySegment s;
  s.h = u.v / u.nq;
  s.first = many_first(u);
  s.j0 = j0;
  s.n = min(u.n - j0, left);
  s.two = u.rows * a.d.G - s.first > 128;
  s.whole = s.n == u.n;
  return s;
}

// A bounded wait that other waits' giving up does not end.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity, uint32_t limit) {
  for (uint32_t i = 0; i < limit && !mbar_try_wait(bar, parity); ++i) __nanosleep(100);
}

// ---- loader -------------------------------------------------------------------------------------------------------------
// The warp's lanes have a block each of four steps: looked up in the table together, asked for in L2 at once, and copied one
// batch later, half a step at a time.  (The ring alone has room for 27 KB on their way, less than memory needs; and one look-up
// after the other took longer than a step.)
template <int Dh>
__device__ void many_load(const AttnArgs& a, ManyShared& sh, unsigned char* raw) {
  using P = ManyPlan<Dh>;
  const ManyPiece piece = copy_of(sh.piece);
  AttnUnit u = piece.u;
  constexpr uint32_t BLK = cache_block_bytes(Dh);
  const int lane = threadIdx.x & 31, per = a.d.ps / CACHE_BLOCK, half_steps = 2 * piece.steps;
  int j = piece.first + (lane >> 3), mine = lane >> 2;   // the lane's step within its unit, its half-step in all
  int page = -1, inner = 0;
  auto look_up = [&]() {
    page = -1;
    if (mine >= half_steps) return;
    while (j >= u.n) { j -= u.n; next_unit<ManyShape>(a, u); }
    const int jb = j * (MANY_TOKENS / CACHE_BLOCK) + (lane & 7), c = jb / per;
    inner = jb - c * per;
    const unsigned last = (unsigned)u.seq + (unsigned)u.rows - 1u;   // the request's last token; a block behind it is not fetched
    if (c < a.d.cols && (unsigned)jb * CACHE_BLOCK <= last) page = __ldg(a.table + (size_t)u.b * a.d.cols + c);
  };
  auto place = [&]() {
    const long long off = block_offset(a.d, page, inner, u.v / u.nq);
    if (off >= 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.pool + off), "r"(BLK) : "memory");
    mine += 8; j += 4;
    return off;
  };
  look_up();
  long long now = place();
  int slot = 0, copied = 0;
  uint32_t phase = 0;
  bool alive = true;
  uint32_t lost = half_steps > 8 ? 0u : a.lost;   // (from the fifth step on where there are more than four)
  while (copied < half_steps && alive) {
    look_up();                       // the next batch's entries are on their way while this one is copied
    const unsigned there8 = __ballot_sync(~0u, now >= 0);
    for (int k = 0; k < 8 && copied < half_steps; ++k, ++copied) {
      const unsigned there = there8 >> (4 * k) & 0xFu;
      if (copied >= MANY_RAW && !__all_sync(~0u, mbar_wait(&sh.bars.raw_free[slot], phase ^ 1u, (volatile int*)&sh.abort, nullptr, a.limit))) { alive = false; break; }
      if (lane == 0) {
        unsigned char* pr = &sh.present[(copied >> 1) % MANY_PRESENT];
        *pr = (unsigned char)((copied & 1) ? *pr | there << 4 : there);
        mbar_expect_tx(&sh.bars.raw_full[slot], __popc(there) * BLK + lost);
      }
      __syncwarp();
      if (lane >> 2 == k && now >= 0)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(smem_u32(raw + slot * P::RAW + (lane & 3) * BLK)), "l"(a.pool + now), "r"(BLK), "r"(smem_u32(&sh.bars.raw_full[slot])) : "memory");
      __syncwarp();
      if (++slot == MANY_RAW) { slot = 0; phase ^= 1u; }
    }
    now = place();
    lost = a.lost;
  }
  // Shared memory is not given up before the last copies have come, whichever wait gives up and when (the last use of a slot completes
  // the phase before the next).
  for (int s = 0; s < MANY_RAW && s < copied; ++s) drain(&sh.bars.raw_full[s], s < slot ? phase : phase ^ 1u, a.limit);
}

// ---- converters ---------------------------------------------------------------------------------------------------------
// A thread's part of 64 raw tokens.  It is read at once, so that the ring's slot is free again before anything is converted.
// K: Dh/8 bytes of the codes of some tokens, with their scales.  A warp's lanes have eight tokens and the four quarters of a row,
// shifted by a quarter every two tokens, so that neither the reads nor the writes of eight lanes meet in a bank.
template <int Dh>
struct KeyPart {
  static constexpr int W = Dh / 32, N = 256 / MANY_CT;
  uint32_t k[N][W], s[N];
  static __device__ __forceinline__ int token(int tid, int n) { return n * (MANY_CT / 4) + (tid >> 5) * 8 + (tid & 7); }
  static __device__ __forceinline__ int quarter(int tid) { return (((tid & 7) >> 1) + ((tid & 31) >> 3)) & 3; }
  __device__ __forceinline__ void read(const unsigned char* raw, int tid) {
    const int q = quarter(tid);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int tok = token(tid, n);
      const unsigned char* blk = raw + (tok >> 4) * cache_block_bytes(Dh);
      const unsigned char* sp = blk + off_ks(Dh) + (tok & 15) * (Dh / CACHE_GROUP) + q * (Dh / 64);
      if (Dh == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(blk + (tok & 15) * (Dh / 2) + q * 16);
        k[n][0] = x.x; k[n][1] = x.y; k[n][W - 2] = x.z; k[n][W - 1] = x.w;
        s[n] = *reinterpret_cast<const unsigned short*>(sp);
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(blk + (tok & 15) * (Dh / 2) + q * 8);
        k[n][0] = x.x; k[n][1] = x.y;
        s[n] = *sp;
      }
    }
  }
  // [token][channel], K-major: rows of 64 channels (128 bytes), 16-byte chunks exchanged by the row's last three bits
  __device__ __forceinline__ void write(unsigned char* dst, int half, int tid) const {
    const int q = quarter(tid);
    unsigned char* at = dst + (q * W >> 3) * ManyPlan<Dh>::SLAB + (half * 64 + token(tid, 0)) * 128;
    uint32_t place[W];
#pragma unroll
    for (int i = 0; i < W; ++i) place[i] = (uint32_t)((((q * W + i) & 7) ^ (tid & 7)) << 4);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const __half2 sc = k_scales(s[n]);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const __half2 ss = Dh == 128 && i >= W / 2 ? __high2half2(sc) : __low2half2(sc);
        uint32_t x[4];
        unpack8(k[n][i], ss, __hmul2(ss, __float2half2_rn(-1032.f)), __hmul2(ss, __float2half2_rn(-72.f)), x);
        *reinterpret_cast<uint4*>(at + n * (MANY_CT / 4) * 128 + place[i]) = make_uint4(x[0], x[1], x[2], x[3]);
      }
    }
  }
};
// V: eight bytes of codes (a group of 16 channels) of Dh/32 tokens, with their scales.
template <int Dh>
struct ValuePart {
  static constexpr int N = 64 * (Dh / CACHE_GROUP) / MANY_CT;
  uint2 v[N]; uint32_t s[N];
  // item: [octet][group][token]
  static __device__ __forceinline__ void item(int tid, int n, int& oct, int& g, int& t8) {
    const int e = tid + n * MANY_CT;
    t8 = e & 7; g = (e >> 3) % (Dh / CACHE_GROUP); oct = (e >> 3) / (Dh / CACHE_GROUP);
  }
  __device__ __forceinline__ void read(const unsigned char* raw, int tid) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      int oct, g, t8;
      item(tid, n, oct, g, t8);
      const unsigned char* b = raw + (oct >> 1) * cache_block_bytes(Dh);
      v[n] = *reinterpret_cast<const uint2*>(b + off_vc(Dh) + (oct & 1) * (4 * Dh) + g * 64 + t8 * 8);
      s[n] = b[off_vs(Dh) + (oct & 1) * (Dh / 2) + g * 8 + t8];
    }
  }
  // [token][channel], MN-major: the same rows; tokens are the contraction
  __device__ __forceinline__ void write(unsigned char* dst, int half, int tid) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      int oct, g, t8;
      item(tid, n, oct, g, t8);
      const int row = half * 64 + oct * 8 + t8;
      const __half2 ss = v_scales(s[n] * 0x101u), c1032 = __hmul2(ss, __float2half2_rn(-1032.f)), c72 = __hmul2(ss, __float2half2_rn(-72.f));
      unsigned char* out = dst + (g >> 2) * ManyPlan<Dh>::SLAB + row * 128;
      uint32_t x[4];
      unpack8(v[n].x, ss, c1032, c72, x);
      *reinterpret_cast<uint4*>(out + ((((g & 3) * 2) ^ (row & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
      unpack8(v[n].y, ss, c1032, c72, x);
      *reinterpret_cast<uint4*>(out + ((((g & 3) * 2 + 1) ^ (row & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
};
// One operand's converters: Part reads and writes it, `full` and `free` are its barriers.
template <class Part, int Dh>
__device__ void many_convert(const AttnArgs& a, ManyShared& sh, unsigned char* raw, unsigned char* stages, uint64_t* full, uint64_t (*free)[2], int tid) {
  using P = ManyPlan<Dh>;
  const ManyPiece piece = copy_of(sh.piece);
  AttnUnit u = piece.u;
  const int lane = threadIdx.x & 31;
  volatile int* abort = (volatile int*)&sh.abort;
  int slot = 0, gj = 0;
  uint32_t phase = 0;
  uint32_t used = 0;   // who read the stages last: bits of groups, by stage
  uint32_t turn = 0;   // parity of the uses so far, a bit for each group and stage
  int left = piece.steps;
  for (int j0 = piece.first; left > 0; j0 = 0) {
    const ManySegment s = many_segment(a, u, j0, left);
    left -= s.n;
#pragma unroll 1
    for (int j = 0; j < s.n; ++j, ++gj) {
      const int st = gj & 1;
      const uint32_t before = used >> (2 * st) & 3u;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        Part part;
        if (!__all_sync(~0u, mbar_wait(&sh.bars.raw_full[slot], phase, abort, nullptr, a.limit))) return;
        part.read(raw + slot * P::RAW, tid);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.bars.raw_free[slot]);
        if (++slot == MANY_RAW) { slot = 0; phase ^= 1u; }
        if (half == 0) {
#pragma unroll
          for (int g = 0; g < 2; ++g)
            if (before >> g & 1u && !__all_sync(~0u, mbar_wait(&free[g][st], (turn >> (2 * st + g) & 1u) ^ 1u, abort, nullptr, a.limit))) return;
        }
        part.write(stages + st * P::TILE, half, tid);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[st]);
      const uint32_t by = s.two ? 3u : 1u << (j & 1);
      used = (used & ~(3u << (2 * st))) | by << (2 * st);
      turn ^= by << (2 * st);
    }
    if (left > 0) next_unit<ManyShape>(a, u);
  }
}

// ---- issuer -------------------------------------------------------------------------------------------------------------
// One thread.  (Tensor memory begins at column 0: all of it is allocated.)  The groups' products are issued in turn, so that
// one group's run while the other has its scores: issued by a thread each they fall into step, and tensor cores and exponentials
// wait for one another.
template <int Dh>
__device__ void many_issue(const AttnArgs& a, ManyShared& sh, unsigned char* smem) {
  using P = ManyPlan<Dh>;
  const ManyPiece piece = copy_of(sh.piece);
  AttnUnit u = piece.u;
  volatile int* abort = (volatile int*)&sh.abort;
  constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(MANY_TOKENS >> 3) << 17) | ((128u >> 4) << 24);              // D = f32, A = B = f16, M = 128; B K-major: keys
  constexpr uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(Dh >> 3) << 17) | ((128u >> 4) << 24);          // B MN-major: values
  const uint64_t qd = smem_desc(smem_u32(smem + P::Q), 16u, 1024u), kd = smem_desc(smem_u32(smem + P::K), 16u, 1024u), vd = smem_desc(smem_u32(smem + P::V), P::SLAB, 1024u);
  uint32_t weights = 0, segments = 0;   // weights: parity of the waits for each group's
  int base = 0;                         // steps before this segment
  int left = piece.steps;
  for (int j0 = piece.first; left > 0; j0 = 0, ++segments) {
    const ManySegment s = many_segment(a, u, j0, left);
    left -= s.n;
    const int ops = s.two ? 2 * s.n : s.n;
    // product i: group i & 1, step i / 2 (two tiles) or i; its P V is issued two products later
#pragma unroll 1
    for (int i = 0; i < ops + 2; ++i) {
      const int g = i & 1;
      // What the two products need besides the weights is waited for first: a wait that finds its barrier complete still takes
      // 200 cycles, and from the weights on everything waits for the products.
      const int jv = base + (s.two ? (i - 2) >> 1 : i - 2), sv = jv & 1, jk = base + (s.two ? i >> 1 : i), sk = jk & 1;
      if (i >= 2 && !mbar_wait(&sh.bars.v_full[sv], (jv >> 1) & 1u, abort, nullptr, a.limit)) return;
      if (i < 2 && i < ops && !mbar_wait(&sh.bars.q_full[g], segments & 1u, abort, nullptr, a.limit)) return;
      if (s.two && i < ops && !mbar_wait(&sh.bars.k_full[sk], (jk >> 1) & 1u, abort, nullptr, a.limit)) return;
      if (i >= 2) {
        if (!mbar_wait(&sh.bars.p_full[g], weights >> g & 1u, abort, nullptr, a.limit)) return;
        weights ^= 1u << g;
      }
      tc_fence_after();
      if (i >= 2) {
        const uint64_t b = vd + (uint64_t)(sv * (P::TILE >> 4));
        const uint32_t more = i >= 4 ? 1u : 0u, o_at = P::O + g * Dh, s_at = g * 128;
#pragma unroll
        for (int ks = 0; ks < MANY_TOKENS / 16; ++ks) mma_tmem_a(o_at, s_at + (ks >> 2) * 64 + (ks & 3) * 8, b + (uint64_t)(ks * 128), id_o, ks > 0 ? 1u : more);
        mma_commit(&sh.bars.o_full[g]);
        mma_commit(&sh.bars.v_free[g][sv]);
      }
      if (i < ops) {
        if (!s.two) {   // (a step's keys are used once here, and not always there in time)
          if (!mbar_wait(&sh.bars.k_full[sk], (jk >> 1) & 1u, abort, nullptr, a.limit)) return;
          tc_fence_after();
        }
        const uint64_t b = kd + (uint64_t)(sk * (P::TILE >> 4)), qa = qd + (uint64_t)(s.two && g ? P::TILE >> 4 : 0);
#pragma unroll
        for (int ks = 0; ks < Dh / 16; ++ks) {
          constexpr uint64_t step = P::SLAB >> 4;
          const uint64_t off = (uint64_t)(ks >> 2) * step + (uint64_t)((ks & 3) * 2);
          mma_bf16(g * 128, qa + off, b + off, id_s, ks > 0 ? 1u : 0u);
        }
        mma_commit(&sh.bars.s_full[g]);
        mma_commit(&sh.bars.k_free[g][sk]);
      }
    }
    base += s.n;
    if (left > 0) next_unit<ManyShape>(a, u);
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

// `count` (a multiple of eight) of a warp's 32 rows of queries, from row `from` on, as fp16 in the operand's layout, times a power of
// two (see Queries in ts_attn.cu): Dh/8 lanes a row and load (a row a lane would touch 32 lines with every load).  f[row]: the
// factor that makes the row's scores exponents of two.  The lane's own row: idx of the unit, `row` of the tile.
template <int Dh>
__device__ __forceinline__ void load_queries(const AttnArgs& a, const AttnUnit& u, int h, int idx, int from, int count, unsigned char* dst, int row, float* f) {
  constexpr int L = Dh / 8, R = 32 / L;   // lanes a row, rows a load
  const int lane = threadIdx.x & 31, c = lane % L, sub = lane / L;
  const long long own = idx < u.rows * a.d.G ? (long long)head_row(a, u.b, h, idx, a.ldq) : -1;
#pragma unroll 1
  for (int k0 = from; k0 < from + count; k0 += 8) {
    uint4 v[8 / R];
#pragma unroll
    for (int k = 0; k < 8 / R; ++k) {
      const long long at = __shfl_sync(~0u, own, k0 + k * R + sub);
      v[k] = at >= 0 ? __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + at) + c) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < 8 / R; ++k) {
      // largest magnitude, as bf16 bits (magnitudes compare as integers)
      uint32_t top = __vmaxu2(__vmaxu2(v[k].x & 0x7FFF7FFFu, v[k].y & 0x7FFF7FFFu), __vmaxu2(v[k].z & 0x7FFF7FFFu, v[k].w & 0x7FFF7FFFu));
#pragma unroll
      for (int x = L / 2; x; x >>= 1) top = __vmaxu2(top, __shfl_xor_sync(~0u, top, x));
      const int e = max((int)(max(top & 0xFFFFu, top >> 16) >> 7), 20);
      // (the sign of the scale goes to the queries: the largest score is the factor times the largest sum)
      const float up = e < 255 ? copysignf(__uint_as_float((unsigned)(127 + 141 - e) << 23), a.qk) : NAN;   // (not finite: NaN, see there)
      const int r = row - lane + k0 + k * R + sub;
      if (c == 0) f[r] = fabsf(a.qk) * __uint_as_float((unsigned)(127 + e - 141) << 23);
      float x[8];
      unpack_bf16x8(v[k], x);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = as_u32(__floats2half2_rn(x[2 * i] * up, x[2 * i + 1] * up));
      *reinterpret_cast<uint4*>(dst + (c >> 3) * ManyPlan<Dh>::SLAB + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}

// n columns of the thread's row in tensor memory times r.  Not often.
__device__ __forceinline__ void scale_columns(uint32_t at, int n, float r) {
#pragma unroll 1
  for (int c = 0; c < n; c += 16) {
    uint32_t x[16];
    tmem_ld16_issue(at + c, x);
    tmem_ld16_wait(x);
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * r);
    tmem_st16(at + c, x);
  }
  tmem_st_wait();
}

// What a softmax thread keeps of its row: weights are 2^(f s - ref), l their sum.  ref moves when a score passes it by ROOM +
// LIFT: weights stay below 2^15, and LIFT keeps small ones out of fp16's subnormals.  References are whole numbers, so that
// what was computed with the old one is taken to the new one without another rounding.
struct SoftRow {
  static constexpr float ROOM = 8.f, LIFT = 7.f;
  float f, m, ref, l;
  // the factor from the old reference to the new one
  __device__ __forceinline__ float move(float top) {
    float r = 1.f;
    if (top > m) {
      const float now = ceilf(top) - LIFT;
      r = m == -INFINITY ? 0.f : ex2(ref - now);
      ref = now; m = now + LIFT + ROOM; l *= r;
    }
    return r;
  }
};

__device__ __forceinline__ float largest(const uint32_t (&x)[32]) {
  float t[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) t[k] = fmaxf(__uint_as_float(x[k]), __uint_as_float(x[k + 4]));
#pragma unroll
  for (int k = 8; k < 32; k += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = fmaxf(t[i], fmaxf(__uint_as_float(x[k + i]), __uint_as_float(x[k + i + 4])));
  return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}

// scores of tokens that the row does not see (bits not set) become -inf
__device__ __forceinline__ void mask_scores(uint32_t (&x)[32], uint32_t on) {
#pragma unroll
  for (int k = 0; k < 32; ++k) x[k] = on >> k & 1u ? x[k] : 0xFF800000u;
}

// 32 scores to fp16 weights: two a fused multiply-add and an addition (f32x2).
__device__ __forceinline__ void weigh(const uint32_t (&x)[32], SoftRow& row, uint32_t (&w)[16]) {
  const uint64_t f2 = pair(row.f, row.f), r2 = pair(-row.ref, -row.ref);
  uint64_t l2 = pair(row.l, 0.f);
#pragma unroll
  for (int k = 0; k < 32; k += 2) {
    float e0, e1;
    unpair(fma2(pair(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, r2), e0, e1);
    e0 = ex2(e0); e1 = ex2(e1);
    l2 = add2(l2, pair(e0, e1));
    w[k / 2] = as_u32(__floats2half2_rn(e0, e1));
  }
  float l0, l1;
  unpair(l2, l0, l1);
  row.l = l0 + l1;
}

template <int Dh>
__device__ void many_softmax(const AttnArgs& a, ManyShared& sh, unsigned char* smem) {
  using P = ManyPlan<Dh>;
  const ManyPiece piece = copy_of(sh.piece);
  AttnUnit u = piece.u;
  volatile int* abort = (volatile int*)&sh.abort;
  // group, half of a step's tokens, row of the tile (a warp reaches the 32 rows of its number modulo 4)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, grp = warp >> 3, hh = (warp >> 2) & 1, quad = warp & 3, row = quad * 32 + lane;
  const uint32_t lanes = (uint32_t)(quad * 32) << 16, ts = lanes + grp * 128 + hh * 64, to = lanes + P::O;
  // the warp's own part of the group's query tile, which results leave through
  unsigned char* stage = smem + P::Q + grp * P::TILE + (Dh == 128 ? hh * P::SLAB + quad * 4096 : quad * 4096 + hh * 2048);
  uint32_t count = 0;   // products of this group
  int base = 0;
  bool alive = true, apart = false;   // apart: the groups had tiles of their own in the unit before
  int left = piece.steps;
  for (int j0 = piece.first; left > 0; j0 = 0) {
    ManySegment s = many_segment(a, u, j0, left);
    left -= s.n;
    int idx = s.first + (s.two ? grp * 128 : 0) + row;
    // The warps of 32 rows load a share each, of their own tile or of the shared one, which the first group's products of the
    // unit before may still read.
    if (!s.two && apart) soft_sync();
    apart = s.two;
    load_queries<Dh>(a, u, s.h, idx, s.two ? 16 * hh : 16 * grp + 8 * hh, s.two ? 16 : 8, smem + P::Q + (s.two ? grp * P::TILE : 0), row, sh.f[s.two ? grp : 0]);
    fence_async_smem();
    if (lane == 0) sh.unit[warp] = u;
    const int seq = u.seq;
    __syncwarp();
    if (lane == 0) {   // (sixteen arrivals: of all warps, or twice of the group's own)
      mbar_arrive(&sh.bars.q_full[grp]);
      mbar_arrive(&sh.bars.q_full[s.two ? grp : grp ^ 1]);
    }
    if (s.two) pair_sync(grp * 4 + quad);
    else soft_sync();
    // (a scale of 0: a factor that makes every finite score 0 and leaves a masked one, -inf, at weight 0)
    SoftRow my{fmaxf(1e-30f, sh.f[s.two ? grp : 0][row]), -INFINITY, 0.f, 0.f};
    int done = 0;   // products of this segment
    // (no way out of the loop: the two warps of 32 rows meet in it, whether or not a wait has given up)
#pragma unroll 1
    for (int j = s.two ? 0 : grp; j < s.n; j += s.two ? 1 : 2) {
      if (alive) alive = __all_sync(~0u, mbar_wait(&sh.bars.s_full[grp], count & 1u, abort, nullptr, a.limit));
      tc_fence_after();
      const int tok0 = (s.j0 + j) * MANY_TOKENS;
      const unsigned here = sh.present[(base + j) % MANY_PRESENT] >> (4 * hh) & 0xFu;
      uint32_t on[2] = {~0u, ~0u}, x[32];
      if (tok0 > seq - MANY_TOKENS || here != 0xFu) {
        const AttnUnit k = copy_of(sh.unit[warp]);
        const int i = tree_row(a, many_first(k) + (s.two ? grp * 128 : 0) + row);
#pragma unroll
        for (int c = 0; c < 2; ++c)
          on[c] = ((here >> (2 * c) & 1u ? 0xFFFFu : 0u) | (here >> (2 * c + 1) & 1u ? 0xFFFF0000u : 0u)) & sees32(a, k.b, i, tok0 + 64 * hh + 32 * c - seq, k.rows);
      }
      float top = -INFINITY;
      if (alive) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          tmem_ld32(ts + 32 * c, x);
          tmem_ld32_wait(x);
          if (__any_sync(~0u, on[c] != ~0u)) mask_scores(x, on[c]);
          top = fmaxf(top, largest(x));
        }
      }
      sh.top[grp][hh][row] = top;
      pair_sync(grp * 4 + quad);
      top = fmaxf(top, sh.top[grp][hh ^ 1][row]) * my.f;
      if (alive && __any_sync(~0u, top > my.m)) {
        const float r = my.move(top);
        if (done > 0) {   // the products before have to be in the sum that is scaled
          alive = __all_sync(~0u, mbar_wait(&sh.bars.o_full[grp], (count - 1u) & 1u, abort, nullptr, a.limit));
          tc_fence_after();
          scale_columns(to + grp * Dh + hh * (Dh / 2), Dh / 2, r);
        }
      }
      if (alive) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t w[16];
          tmem_ld32(ts + 32 * c, x);
          tmem_ld32_wait(x);
          if (__any_sync(~0u, on[c] != ~0u)) mask_scores(x, on[c]);
          weigh(x, my, w);
          tmem_st16(ts + 16 * c, w);   // (the weights replace scores that are taken)
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.bars.p_full[grp]);
      }
      ++count;
      ++done;
    }
    // ---- results: by group and half, channels of the group's own tile or of the rows that the groups share
    u = copy_of(sh.unit[warp]);
    s = many_segment(a, u, j0, s.n);
    idx = s.first + (s.two ? grp * 128 : 0) + row;
    if (alive && done > 0) alive = __all_sync(~0u, mbar_wait(&sh.bars.o_full[grp], (count - 1u) & 1u, abort, nullptr, a.limit));
    sh.top[grp][hh][row] = my.m == -INFINITY ? -INFINITY : my.ref;
    sh.sum[grp][hh][row] = my.l;
    if (s.two) pair_sync(grp * 4 + quad);
    else soft_sync();         // (both groups' products are complete: each has waited for its own)
    float sum, top, w0 = 1.f, w1 = 0.f;   // weights of the groups' parts
    if (s.two) {
      top = sh.top[grp][0][row];
      sum = sh.sum[grp][0][row] + sh.sum[grp][1][row];
    } else {
      const float t0 = sh.top[0][0][row], t1 = sh.top[1][0][row];
      top = fmaxf(t0, t1);
      w0 = part_weight(t0, top); w1 = part_weight(t1, top);
      sum = w0 * (sh.sum[0][0][row] + sh.sum[0][1][row]) + w1 * (sh.sum[1][0][row] + sh.sum[1][1][row]);
    }
    const bool other = !s.two && s.n > 1;   // (with one step the second group's sum was never written)
    if (!alive || *abort) sum = NAN;
    tc_fence_after();
    const int rows = u.rows * a.d.G;
    const int slot = ((int)blockIdx.x * 2 + (s.j0 > 0 ? 0 : 1)) * MANY_QT + (s.two ? grp * 128 : 0) + row;
    const float inv = s.whole ? row_inv(sum) * a.vo : 1.f;
    const int n = s.two ? Dh / 64 : 1, c_lo = (s.two ? hh : grp * 2 + hh) * n, c_hi = min(c_lo + n, Dh / 32);   // groups of 32 channels
    if (idx < rows && hh == 0 && (s.two || grp == 0)) {
      if (!s.whole) { a.part_ml[2 * slot] = top; a.part_ml[2 * slot + 1] = sum; }
      else if (a.lse) a.lse[lse_row(a, u.b, s.h, idx)] = row_lse(top, sum);
    }
    // through the stage in pieces of 16 bytes, so that rows leave in whole lines: 32 channels as bf16 or fp32, 16 as fp32 where a
    // staged row has no more room
    constexpr int ROOM = Dh / 16;   // pieces of a staged row
    const int bits = s.whole || ROOM == 4 ? 2 : 3;
    const bool halves = !s.whole && ROOM == 4;
#pragma unroll 1
    for (int c = 2 * c_lo; c < 2 * c_hi; ++c) {   // (16 channels at a time: 32 with the other group's do not fit the registers)
      uint32_t x[16];
      tmem_ld16_issue(to + (s.two ? grp * Dh : 0) + 16 * c, x);
      tmem_ld16_wait(x);
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(w0 * __uint_as_float(x[k]) * inv);
      if (other) {
        uint32_t y[16];
        tmem_ld16_issue(to + Dh + 16 * c, y);
        tmem_ld16_wait(y);
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(fmaf(w1 * inv, __uint_as_float(y[k]), __uint_as_float(x[k])));
      }
      auto put = [&](int k, uint4 v) { *reinterpret_cast<uint4*>(stage + lane * Dh + ((k ^ (lane & (ROOM - 1))) << 4)) = v; };
      if (s.whole) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const __nv_bfloat162 h2 = __floats2bfloat162_rn(__uint_as_float(x[8 * k + 2 * q]), __uint_as_float(x[8 * k + 2 * q + 1]));
            w[q] = *reinterpret_cast<const uint32_t*>(&h2);
          }
          put(2 * (c & 1) + k, make_uint4(w[0], w[1], w[2], w[3]));
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) put((4 * (c & 1) + k) & (ROOM - 1), make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]));
      }
      if (!halves && !(c & 1)) continue;
      __syncwarp();
      const int ch = halves ? 16 * c : 16 * (c & ~1);   // the first staged channel
      for (int e = lane; e < 32 << bits; e += 32) {
        const int r = e >> bits, k = e - (r << bits), id = idx - lane + r;
        if (id >= rows) break;   // (rows rise with e)
        const uint4 t = *reinterpret_cast<const uint4*>(stage + r * Dh + ((k ^ (r & (ROOM - 1))) << 4));
        if (s.whole) reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + out_row(a, u.b, s.h, id) + ch)[k] = t;
        else reinterpret_cast<uint4*>(a.part + (size_t)(slot - lane + r) * Dh + ch)[k] = t;
      }
      __syncwarp();
    }
    tc_fence_before();
    // all have read the sums and left the stages, before the next unit's products and queries overwrite them
    if (s.two) pair_sync(grp * 4 + quad);
    else soft_sync();
    base += s.n;
    if (left > 0) next_unit<ManyShape>(a, u);
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
      mbar_init(&b.k_full[s], MANY_CONV / 2); mbar_init(&b.k_free[0][s], 1); mbar_init(&b.k_free[1][s], 1);
      mbar_init(&b.v_full[s], MANY_CONV / 2); mbar_init(&b.v_free[0][s], 1); mbar_init(&b.v_free[1][s], 1);
      mbar_init(&b.q_full[s], MANY_SOFT); mbar_init(&b.s_full[s], 1); mbar_init(&b.p_full[s], MANY_SOFT / 2); mbar_init(&b.o_full[s], 1);
    }
    mbar_init(&b.issued, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  AttnUnit u;
  int first;
  long long steps;
  if (!attn_locate<ManyShape, MANY_THREADS>(a, u, first, steps)) return;
  if (warp == MANY_ISSUE) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) { sh.piece.u = u; sh.piece.first = first; sh.piece.steps = (int)steps; }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (sh.tmem != 0u) sh.abort = 1;   // (cannot be: 512 columns were asked for)
  bool issuer = false;
  if (warp < MANY_SOFT) {
    many_softmax<Dh>(a, sh, smem);
  } else {
    if (warp < MANY_SOFT + MANY_CONV / 2)
      many_convert<KeyPart<Dh>, Dh>(a, sh, smem + P::R, smem + P::K, sh.bars.k_full, sh.bars.k_free, threadIdx.x - MANY_SOFT * 32);
    else if (warp < MANY_ISSUE)
      many_convert<ValuePart<Dh>, Dh>(a, sh, smem + P::R, smem + P::V, sh.bars.v_full, sh.bars.v_free, threadIdx.x - MANY_SOFT * 32 - MANY_CT);
    else if (warp == MANY_ISSUE) {
      if (elect_one()) {
        many_issue<Dh>(a, sh, smem);
        issuer = true;
      }
    }
    else if (warp == MANY_LOAD) many_load<Dh>(a, sh, smem + P::R);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Nor is tensor memory given up before the last products are complete.  (Without a wait that gave up the softmax warps have waited for them.)
  if (issuer && sh.abort) {
    mma_commit(&sh.bars.issued);
    drain(&sh.bars.issued, 0u, a.limit);
  }
  __syncwarp();
  if (warp == MANY_ISSUE) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(512u) : "memory");
}

static_assert(sizeof(ManyShared) + ManyPlan<128>::SMEM + 128 <= 227 * 1024, "shared memory");

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

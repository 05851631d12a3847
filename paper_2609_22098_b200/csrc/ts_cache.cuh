// The 4-bit key/value cache: layout, argument checks and the pieces that its kernels share.
//
// A layer's pool is [n_pages][Hkv][page_size / 16][18 * Dh] bytes.  A block = 16 tokens of one head, contiguous, so that a
// kernel fetches it with one bulk copy whatever the page size:
//   K codes [16][Dh/2] | V codes [2][Dh/16][8][8 bytes] | K scales [16][Dh/16] | V scales [2][Dh/16][8]
// V lies group by group within octets of tokens: a lane of a matrix instruction needs a few channels of token pairs, and
// finds them in 16 consecutive bytes (row by row, its reads would meet in the same banks four at a time).
// A code c in 0..15 and its group's e4m3 scale s stand for (c - 8) * s * 2^exp.  Eight elements share a 32-bit word: element
// 2j is nibble j, element 2j + 1 nibble j + 4, so that a mask leaves neighbouring elements in the two halves of a word.
#pragma once

#include <cuda_fp16.h>

#include "ts_internal.h"

namespace ts {

constexpr int CACHE_BLOCK = 16;    // tokens of a block
constexpr int CACHE_GROUP = 16;    // elements that share a scale
constexpr unsigned SCALE_NAN = 0x7Fu;

__host__ __device__ constexpr int cache_block_bytes(int Dh) { return 18 * Dh; }
__host__ __device__ constexpr int off_vc(int Dh) { return 8 * Dh; }
__host__ __device__ constexpr int off_ks(int Dh) { return 16 * Dh; }
__host__ __device__ constexpr int off_vs(int Dh) { return 17 * Dh; }

// sizes that the kernels index with
struct CacheDims {
  int Hq, Hkv, G, Dh, ps, n_pages, cols;   // G = query heads of a kv head; cols = columns of the block table
  __host__ __device__ size_t page_bytes() const { return (size_t)Hkv * (ps / CACHE_BLOCK) * cache_block_bytes(Dh); }
};

// NULL: fine; else what is wrong
const char* cache_layout_error(const ts_cache_layout* lay);
int32_t set_layout_error(const char* call, const ts_cache_layout* lay);
CacheDims cache_dims(const ts_cache_layout* lay);
// the device that a context belongs to has to be the current one
bool on_ctx_device(const ts_ctx* ctx);

inline bool bad_ptr4(const void* p) { return !p || ((uintptr_t)p & 3u); }

// Rows of a request: the anchor and its nodes.  A negative length: the request takes no part.
__device__ __forceinline__ int request_rows(const int* n_nodes, int b, int rcap) {
  return n_nodes ? min(max(n_nodes[b], 0), rcap - 1) + 1 : 1;
}

// Byte address of block `inner` of a page for head h, -1 where the table's entry is no page.
__device__ __forceinline__ long long block_offset(const CacheDims& d, int page, int inner, int h) {
  if ((unsigned)page >= (unsigned)d.n_pages) return -1;
  const unsigned per = d.ps / CACHE_BLOCK;   // (a page has less than 2^32 bytes: 1,024 heads, 4,096 tokens, 144 bytes each)
  return ((long long)((unsigned long long)(unsigned)page * ((unsigned)d.Hkv * per)) + (unsigned)h * per + (unsigned)inner) * cache_block_bytes(d.Dh);
}

// Eight codes of a word as four half2 of (c - 8) * s, times the power of two that s carries: h[j] = elements 2j, 2j + 1.
// The code is put into the mantissa of 1024 (nibble at bit 0) or 64 (nibble at bit 4); one fused multiply-add takes that off
// and scales.  Exact: s has four significant bits, 1032 s at most 11 (129 * 15 < 2048) and (c - 8) s at most eight.
__device__ __forceinline__ void unpack8(uint32_t w, __half2 s, __half2 s1032, __half2 s72, uint32_t* h) {
  uint32_t x0, x1, x2, x3;
  const uint32_t w8 = w >> 8;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x0) : "r"(w));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x54005400, 0xEA;" : "=r"(x1) : "r"(w));
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x2) : "r"(w8));
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x54005400, 0xEA;" : "=r"(x3) : "r"(w8));
  const __half2 r0 = __hfma2(*reinterpret_cast<__half2*>(&x0), s, s1032), r1 = __hfma2(*reinterpret_cast<__half2*>(&x1), s, s72);
  const __half2 r2 = __hfma2(*reinterpret_cast<__half2*>(&x2), s, s1032), r3 = __hfma2(*reinterpret_cast<__half2*>(&x3), s, s72);
  h[0] = *reinterpret_cast<const uint32_t*>(&r0); h[1] = *reinterpret_cast<const uint32_t*>(&r1);
  h[2] = *reinterpret_cast<const uint32_t*>(&r2); h[3] = *reinterpret_cast<const uint32_t*>(&r3);
}

__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t as_u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }

// Two e4m3 scales of K as fp16, times 2^-3 (so that 1032 s stays below 65,504).  NaN stays NaN: what is scored with it is too.
constexpr int K_SHIFT = 3;
__device__ __forceinline__ __half2 k_scales(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  return __hmul2(as_half2(r), __float2half2_rn(0.125f));
}
// Two e4m3 scales of V as fp16, times 2^-8: the byte moved into place.  Never NaN or infinite, so that a token of weight
// zero adds zero whatever its bytes are; a token that holds NaN has NaN scales of K too and gives its rows NaN by those.
constexpr int V_SHIFT = 8;
__device__ __forceinline__ __half2 v_scales(uint32_t two) { return as_half2((__byte_perm(two, 0u, 0x4140) & 0x007F007Fu) << 7); }

}  // namespace ts

// The paged key/value cache as the kernels see it, and its 8-bit format.
#pragma once

#include "fox_device.h"
#include "fox_internal.h"

namespace fox {

// k, v [n_pages][Hkv][page][d] in the cache's type, for e4m3 the rows' scales ke, ve
// [n_pages][Hkv][page], c [n_pages][H][page] fp32; table [B][max_pages].
struct CacheView {
  void* k;
  void* v;
  uint8_t* ke;
  uint8_t* ve;
  float* c;
  const int* table;
  int n_pages, page_shift, max_pages, B, H, Hkv;

  __device__ long long capacity() const { return (long long)max_pages << page_shift; }
  // The page that holds position pos of sequence b; -1 where the table has no page for it
  // or names one that does not exist.  Nothing is read or written through a -1.
  __device__ int page_of(int b, int pos) const {
    const int i = pos >> page_shift;
    if (pos < 0 || i >= max_pages) return -1;
    const int p = table[(size_t)b * max_pages + i];
    return (unsigned)p < (unsigned)n_pages ? p : -1;
  }
  // The table's entry for position pos (outside the table, of its nearest place), unchecked, by
  // a scalar load: pos is the same in the whole wave.  page_exists() says whether it is a page.
  __device__ int page_entry(int b, int pos) const {
    typedef const __attribute__((address_space(4))) int table_t;
    const int i = min(max(pos, 0) >> page_shift, max_pages - 1);
    return ((table_t*)(uintptr_t)table)[(size_t)b * max_pages + i];
  }
  __device__ bool page_exists(int p) const { return (unsigned)p < (unsigned)n_pages; }
  __device__ int slot_of(int pos) const { return pos & ((1 << page_shift) - 1); }
  // index of (page p, key head h, slot) in k_exp and, times d, in k and v
  __device__ size_t kv_row(int p, int h, int slot) const {
    return (((size_t)p * Hkv + h) << page_shift) + slot;
  }
  __device__ size_t c_at(int p, int h, int slot) const {
    return (((size_t)p * H + h) << page_shift) + slot;
  }
};

inline CacheView cache_view(const CacheSpec& s) {
  return CacheView{s.k,       s.v,      s.k_exp,     s.v_exp, s.c, s.page_table, s.n_pages,
                   __builtin_ctz((unsigned)s.page), s.max_pages, s.B,   s.H, s.Hkv};
}

constexpr int kMaxNew = 64;  // new tokens of a sequence per call: a row's ancestors are 64 bits

// A buffer descriptor whose parts are the same in the whole wave but that the compiler cannot
// see to be (it would loop over the lanes' descriptors around every load).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const char* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const uint64_t u = ((uint64_t)uniform_u32((uint32_t)(a >> 32)) << 32) | uniform_u32((uint32_t)a);
  return make_rsrc((const void*)(uintptr_t)u, uniform_u32(bytes));
}

// e4m3 rows share one scale 2^e, stored as the biased exponent e + 127.  It is the least
// power of two, from 2^-126, that brings the row's largest magnitude to 448 or below.  A
// power of two costs a floating-point code no accuracy (only its subnormal end moves), it
// makes the division exact, and code * 2^e is exact in bf16 (four significant bits).
// With amax = 1.m * 2^(E - 127) and 448 = 1.75 * 2^8: e = E - 127 - 8, one more if 1.m > 1.75.
__device__ __forceinline__ uint32_t e4m3_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float e4m3_scale(uint32_t biased) { return __uint_as_float(biased << 23); }
__device__ __forceinline__ float e4m3_inverse(uint32_t biased) {
  return __uint_as_float((254u - biased) << 23);
}

// four e4m3 codes times a power of two to bf16
__device__ __forceinline__ void e4m3_to_bf16(uint32_t w, float scale, bf16x2& lo, bf16x2& hi) {
  lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
}
// eight consecutive codes as one MFMA operand
__device__ __forceinline__ bf16x8 e4m3_operand(uint32_t a, uint32_t b, float scale) {
  bf16x2 p[4];
  e4m3_to_bf16(a, scale, p[0], p[1]);
  e4m3_to_bf16(b, scale, p[2], p[3]);
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = p[i][0];
    r[2 * i + 1] = p[i][1];
  }
  return r;
}

}  // namespace fox

// The paged key/value cache: new tokens quantised as they are written, accepted drafts moved
// together, positions read back.
//
//   append         k, v [B,Hkv,n,d] and the gate logits [B,H,n] of up to 64 new tokens per
//                  sequence, a chain or a tree: c of a token is c of the token it follows plus
//                  log sigmoid(logit), the token it follows being its parent among the new
//                  ones or the last cached one.
//   append_packed  k, v [Hkv,N,d] and c [H,N] of whole prompts (cu_seqlens), behind what each
//                  sequence has in the cache.
//   keep           rows seq_len + index[j] move to seq_len + j (an accepted path of a tree).
//   read           positions start .. of each sequence as bf16 or fp32 (code times scale:
//                  exact in both).
//
// All of them are bound by the rows' bytes, and at small sizes by the launch: 36 thousand prompt
// tokens of H = 16, H_kv = 4, d = 128, bf16 to e4m3, are written in 27 us (119 MB, 4.4 TB/s) and read
// back in 21 us (120 MB, 5.8 TB/s; a plain copy reaches 4.8); one token of each of 64 sequences
// takes 3.6 us.  D / 8 lanes
// share a row, eight elements each: 16 bytes of bf16 in, 8 bytes of codes out; the row's
// largest magnitude meets over DPP.  Each call is one launch: the first workgroups take the
// prefix values, the rest the rows.  Rows and values are counted in 32 bits (their products
// with the heads are below 2^31), their bytes in 64.
#include "fox_internal.h"
#include "kv_cache.h"

namespace fox {

constexpr int kCacheThreads = 256;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4c __attribute__((ext_vector_type(4)));

// maximum over aligned groups of 8 or 16 lanes, in every lane
template <int LPR>
__device__ __forceinline__ float row_max(float x) {
  static_assert(LPR == 8 || LPR == 16, "rows span 8 or 16 lanes");
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  x = fmaxf(x, dpp<0x141>(x));
  if constexpr (LPR == 16) x = fmaxf(x, dpp<0x140>(x));
  return x;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_f32(v[e]);
  } else {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = a[e];
      x[4 + e] = b[e];
    }
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<bf16x8*>(p) = pack8(x);
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Lane `part` of a row's D / 8 lanes writes its eight elements to cache row `row`.  Values
// that are not finite become NaN codes and do not take part in the scale.
template <int D, bool F8>
__device__ __forceinline__ void put_row(void* dst, uint8_t* exps, size_t row, int part,
                                        float (&x)[8]) {
  if constexpr (F8) {
    float amax = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = fabsf(x[e]);
      if (a < INFINITY) amax = fmaxf(amax, a);
      else x[e] = __uint_as_float(0x7fc00000u);
    }
    const uint32_t ex = e4m3_exponent(row_max<D / 8>(amax));
    const float inv = e4m3_inverse(ex);
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, c, true);
      w[i] = (uint32_t)c;
    }
    *reinterpret_cast<u32x2*>(static_cast<char*>(dst) + row * D + 8 * part) = w;
    if (part == 0) exps[row] = (uint8_t)ex;
  } else {
    store8(static_cast<bf16*>(dst) + row * D + 8 * part, x);
  }
}

// c of the last cached token (0 before the first)
__device__ __forceinline__ float cached_c(const CacheView& cv, int b, int h, int len) {
  const int p = cv.page_of(b, len - 1);
  return p < 0 ? 0.0f : cv.c[cv.c_at(p, h, cv.slot_of(len - 1))];
}

// ---------------------------------------------------------------------------
// append: gate_groups workgroups of four (sequence, head) waves, then the rows
// ---------------------------------------------------------------------------
template <typename T, int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void cache_append_kernel(
    CacheView cv, const T* __restrict__ k, const T* __restrict__ v,
    const float* __restrict__ logit, const int* __restrict__ seq_len,
    const int* __restrict__ parent, const int* __restrict__ n_new, int n, unsigned gate_groups) {
  if (blockIdx.x < gate_groups) {
    // lane = new token: c = c_cached + the sum of log f over its ancestors and itself, by
    // doubling pointers, in 64 bits and rounded once
    const int lane = threadIdx.x & 63;
    const unsigned job = blockIdx.x * (kCacheThreads / 64) + (threadIdx.x >> 6);
    if (job >= (unsigned)(cv.B * cv.H)) return;
    const int b = (int)(job / cv.H), h = (int)(job % cv.H);
    const int len = max(seq_len[b], 0), nn = n_new ? min(n_new[b], n) : n;
    double sum = 0.0;
    int up = -1;
    if (lane < nn) {
      sum = log_sigmoid(logit[(size_t)job * n + lane]);
      up = parent ? parent[(size_t)b * n + lane] : lane - 1;
      if (up >= lane) up = -1;
    }
    while (__any(up >= 0)) {
      const int from = up >= 0 ? up : lane;
      const double s = __shfl(sum, from);
      const int u = __shfl(up, from);
      if (up >= 0) {
        sum += s;
        up = u;
      }
    }
    if (lane < nn && len <= cv.capacity() - 1 - lane) {
      const int p = cv.page_of(b, len + lane);
      if (p >= 0) cv.c[cv.c_at(p, h, cv.slot_of(len + lane))] = (float)(cached_c(cv, b, h, len) + sum);
    }
    return;
  }
  constexpr int LPR = D / 8, RPB = kCacheThreads / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned r = (blockIdx.x - gate_groups) * RPB + threadIdx.x / LPR;
  if (r >= (unsigned)(cv.B * cv.Hkv * n)) return;  // whole rows leave together
  // the row first: its loads are under way while its place is looked up
  float x[8], y[8];
  load8(k + (size_t)r * D + 8 * part, x);
  load8(v + (size_t)r * D + 8 * part, y);
  const unsigned bh = r / n;
  const int t = (int)(r % n), h = (int)(bh % cv.Hkv), b = (int)(bh / cv.Hkv);
  const int len = max(seq_len[b], 0), nn = n_new ? min(n_new[b], n) : n;
  if (t >= nn || len > cv.capacity() - 1 - t) return;
  const int p = cv.page_of(b, len + t);
  if (p < 0) return;
  const size_t row = cv.kv_row(p, h, cv.slot_of(len + t));
  put_row<D, F8>(cv.k, cv.ke, row, part, x);
  put_row<D, F8>(cv.v, cv.ve, row, part, y);
}

// ---------------------------------------------------------------------------
// append_packed
// ---------------------------------------------------------------------------
// The sequence that packed row r belongs to (the last one that starts at or before it); rows
// before the first or behind the last sequence give -1.
__device__ __forceinline__ int packed_sequence(const int* __restrict__ cu, int B, int r) {
  int lo = 0, hi = B;  // cu[lo] <= r < cu[hi]
  if (r < cu[0] || r >= cu[B]) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <typename T, int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void cache_append_packed_kernel(
    CacheView cv, const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ c,
    const int* __restrict__ cu, const int* __restrict__ seq_len, int N, unsigned gate_groups) {
  if (blockIdx.x < gate_groups) {
    const unsigned i = blockIdx.x * kCacheThreads + threadIdx.x;
    if (i >= (unsigned)(cv.H * N)) return;
    const int h = (int)(i / N), r = (int)(i % N);
    const int b = packed_sequence(cu, cv.B, r);
    if (b < 0) return;
    const int len = seq_len ? max(seq_len[b], 0) : 0, t = r - cu[b];
    if (len > cv.capacity() - 1 - t) return;
    const int p = cv.page_of(b, len + t);
    if (p >= 0) cv.c[cv.c_at(p, h, cv.slot_of(len + t))] = cached_c(cv, b, h, len) + c[i];
    return;
  }
  constexpr int LPR = D / 8, RPB = kCacheThreads / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned i = (blockIdx.x - gate_groups) * RPB + threadIdx.x / LPR;
  if (i >= (unsigned)(cv.Hkv * N)) return;
  float x[8], y[8];  // the row first, as above
  load8(k + (size_t)i * D + 8 * part, x);
  load8(v + (size_t)i * D + 8 * part, y);
  const int h = (int)(i / N), r = (int)(i % N);
  const int b = packed_sequence(cu, cv.B, r);
  if (b < 0) return;
  const int len = seq_len ? max(seq_len[b], 0) : 0, t = r - cu[b];
  if (len > cv.capacity() - 1 - t) return;
  const int p = cv.page_of(b, len + t);
  if (p < 0) return;
  const size_t row = cv.kv_row(p, h, cv.slot_of(len + t));
  put_row<D, F8>(cv.k, cv.ke, row, part, x);
  put_row<D, F8>(cv.v, cv.ve, row, part, y);
}

// ---------------------------------------------------------------------------
// keep: one workgroup per (sequence, key head) moves its rows of k and v, one per (sequence,
// head) the prefix values.  Everything that a workgroup moves is in registers before it
// stores any, so sources and destinations may overlap in any order.
// ---------------------------------------------------------------------------
template <int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void cache_keep_kernel(
    CacheView cv, const int* __restrict__ seq_len, const int* __restrict__ index,
    const int* __restrict__ n_keep, int n) {
  __shared__ int src_page[kMaxNew], dst_page[kMaxNew], src_slot[kMaxNew], dst_slot[kMaxNew];
  const int b = (int)(blockIdx.x / (cv.Hkv + cv.H)), part = (int)(blockIdx.x % (cv.Hkv + cv.H));
  const int len = max(seq_len[b], 0), m = max(0, min(n_keep[b], n));
  const int tid = threadIdx.x;
  if (tid < m) {
    const int from = index[(size_t)b * n + tid];
    int sp = -1, dp = -1;
    // a draft's place is one of the 64 behind seq_len
    if (from >= 0 && from < kMaxNew) {
      if (len <= cv.capacity() - 1 - from) sp = cv.page_of(b, len + from);
      if (len <= cv.capacity() - 1 - tid) dp = cv.page_of(b, len + tid);
    }
    if (sp < 0) dp = -1;
    src_page[tid] = sp;
    dst_page[tid] = dp;
    src_slot[tid] = cv.slot_of(len + max(from, 0));
    dst_slot[tid] = cv.slot_of(len + tid);
  }
  __syncthreads();
  if (part >= cv.Hkv) {
    const int h = part - cv.Hkv;
    float x = 0.0f;
    const bool ok = tid < m && dst_page[tid] >= 0;
    if (ok) x = cv.c[cv.c_at(src_page[tid], h, src_slot[tid])];
    __syncthreads();
    if (ok) cv.c[cv.c_at(dst_page[tid], h, dst_slot[tid])] = x;
    return;
  }
  constexpr int CPR = D * (F8 ? 1 : 2) / 16;                  // 16-byte pieces of a row
  constexpr int PER = kMaxNew * CPR / kCacheThreads;          // of each thread, k and v each
  static_assert(PER * kCacheThreads == kMaxNew * CPR, "the threads cover 64 rows exactly");
  u32x4c xk[PER], xv[PER];
  uint8_t ek = 0, ev = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int piece = i * kCacheThreads + tid, j = piece / CPR;
    if (j < m && dst_page[j] >= 0) {
      const size_t at = cv.kv_row(src_page[j], part, src_slot[j]) * CPR + piece % CPR;
      xk[i] = static_cast<const u32x4c*>(cv.k)[at];
      xv[i] = static_cast<const u32x4c*>(cv.v)[at];
    }
  }
  const bool eo = F8 && tid < m && dst_page[tid] >= 0;
  if (eo) {
    const size_t at = cv.kv_row(src_page[tid], part, src_slot[tid]);
    ek = cv.ke[at];
    ev = cv.ve[at];
  }
  __syncthreads();  // (waits for the loads of every wave)
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int piece = i * kCacheThreads + tid, j = piece / CPR;
    if (j < m && dst_page[j] >= 0) {
      const size_t at = cv.kv_row(dst_page[j], part, dst_slot[j]) * CPR + piece % CPR;
      static_cast<u32x4c*>(cv.k)[at] = xk[i];
      static_cast<u32x4c*>(cv.v)[at] = xv[i];
    }
  }
  if (eo) {
    const size_t at = cv.kv_row(dst_page[tid], part, dst_slot[tid]);
    cv.ke[at] = ek;
    cv.ve[at] = ev;
  }
}

// ---------------------------------------------------------------------------
// read
// ---------------------------------------------------------------------------
template <typename T, int D, bool F8>
__device__ __forceinline__ void get_row(const void* src, const uint8_t* exps, size_t row, int part,
                                        T* out) {
  float x[8];
  if constexpr (F8) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const char*>(src) + row * D + 8 * part);
    const float s = e4m3_scale(exps[row]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      x[4 * i] = lo[0] * s;
      x[4 * i + 1] = lo[1] * s;
      x[4 * i + 2] = hi[0] * s;
      x[4 * i + 3] = hi[1] * s;
    }
  } else {
    load8(static_cast<const bf16*>(src) + row * D + 8 * part, x);
  }
  store8(out, x);
}

template <typename T, int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(
    CacheView cv, const int* __restrict__ start, const int* __restrict__ seq_len,
    T* __restrict__ k, T* __restrict__ v, float* __restrict__ c, int T_, bool zero_others,
    unsigned gate_groups) {
  // the page of row t of sequence b, -1 where it has no token
  auto page = [&](int b, int t, int& slot) {
    const int s0 = start ? max(start[b], 0) : 0;
    slot = cv.slot_of(s0 + t);
    return t < max(seq_len[b], 0) - s0 ? cv.page_of(b, s0 + t) : -1;
  };
  int slot;
  if (blockIdx.x < gate_groups) {
    const unsigned i = blockIdx.x * kCacheThreads + threadIdx.x, bh = i / T_;
    if (i >= (unsigned)(cv.B * cv.H * T_)) return;
    const int t = (int)(i % T_), h = (int)(bh % cv.H), b = (int)(bh / cv.H);
    const int p = page(b, t, slot);
    if (p >= 0) c[i] = cv.c[cv.c_at(p, h, slot)];
    else if (zero_others) c[i] = 0.0f;
    return;
  }
  constexpr int LPR = D / 8, RPB = kCacheThreads / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned r = (blockIdx.x - gate_groups) * RPB + threadIdx.x / LPR, bh = r / T_;
  if (r >= (unsigned)(cv.B * cv.Hkv * T_)) return;
  const int t = (int)(r % T_), h = (int)(bh % cv.Hkv), b = (int)(bh / cv.Hkv);
  const int p = page(b, t, slot);
  T *ko = k + (size_t)r * D + 8 * part, *vo = v + (size_t)r * D + 8 * part;
  if (p >= 0) {
    const size_t row = cv.kv_row(p, h, slot);
    get_row<T, D, F8>(cv.k, cv.ke, row, part, ko);
    get_row<T, D, F8>(cv.v, cv.ve, row, part, vo);
  } else if (zero_others) {
    const float zeros[8] = {};
    store8(ko, zeros);
    store8(vo, zeros);
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
static unsigned groups_of(long long jobs, int per) { return (unsigned)((jobs + per - 1) / per); }

// f(type tag, std::integral_constant<int, D>, std::bool_constant<F8>)
template <typename F>
static void cache_dispatch(const CacheSpec& s, bool bf16_, F&& f) {
  auto by_format = [&](auto tag, auto dc) {
    if (s.f8) f(tag, dc, std::true_type());
    else f(tag, dc, std::false_type());
  };
  auto by_dim = [&](auto tag) {
    if (s.d == 128) by_format(tag, std::integral_constant<int, 128>());
    else by_format(tag, std::integral_constant<int, 64>());
  };
  if (bf16_) by_dim((bf16*)nullptr);
  else by_dim((float*)nullptr);
}

hipError_t launch_cache_append(const CacheSpec& s, bool bf16_, const void* k, const void* v,
                               const float* logit, const int* seq_len, const int* parent,
                               const int* n_new, int n, hipStream_t st) {
  const unsigned gates = groups_of((long long)s.B * s.H, kCacheThreads / 64);
  const unsigned rows = groups_of((long long)s.B * s.Hkv * n, kCacheThreads / (s.d / 8));
  cache_dispatch(s, bf16_, [&](auto tag, auto dc, auto f8) {
    typedef std::remove_pointer_t<decltype(tag)> T;
    hipLaunchKernelGGL((cache_append_kernel<T, decltype(dc)::value, decltype(f8)::value>),
                       dim3(gates + rows), dim3(kCacheThreads), 0, st, cache_view(s), (const T*)k,
                       (const T*)v, logit, seq_len, parent, n_new, n, gates);
  });
  return hipGetLastError();
}

hipError_t launch_cache_append_packed(const CacheSpec& s, bool bf16_, const void* k, const void* v,
                                      const float* c, const int* cu, const int* seq_len, int N,
                                      hipStream_t st) {
  const unsigned gates = groups_of((long long)s.H * N, kCacheThreads);
  const unsigned rows = groups_of((long long)s.Hkv * N, kCacheThreads / (s.d / 8));
  cache_dispatch(s, bf16_, [&](auto tag, auto dc, auto f8) {
    typedef std::remove_pointer_t<decltype(tag)> T;
    hipLaunchKernelGGL((cache_append_packed_kernel<T, decltype(dc)::value, decltype(f8)::value>),
                       dim3(gates + rows), dim3(kCacheThreads), 0, st, cache_view(s), (const T*)k,
                       (const T*)v, c, cu, seq_len, N, gates);
  });
  return hipGetLastError();
}

hipError_t launch_cache_keep(const CacheSpec& s, const int* seq_len, const int* index,
                             const int* n_keep, int n, hipStream_t st) {
  const unsigned groups = (unsigned)s.B * (unsigned)(s.Hkv + s.H);
  cache_dispatch(s, true, [&](auto, auto dc, auto f8) {
    hipLaunchKernelGGL((cache_keep_kernel<decltype(dc)::value, decltype(f8)::value>), dim3(groups),
                       dim3(kCacheThreads), 0, st, cache_view(s), seq_len, index, n_keep, n);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheSpec& s, bool bf16_, const int* start, const int* seq_len,
                             void* k, void* v, float* c, int T_, bool zero_others, hipStream_t st) {
  const unsigned gates = c ? groups_of((long long)s.B * s.H * T_, kCacheThreads) : 0;
  const unsigned rows = groups_of((long long)s.B * s.Hkv * T_, kCacheThreads / (s.d / 8));
  cache_dispatch(s, bf16_, [&](auto tag, auto dc, auto f8) {
    typedef std::remove_pointer_t<decltype(tag)> T;
    hipLaunchKernelGGL((cache_read_kernel<T, decltype(dc)::value, decltype(f8)::value>),
                       dim3(gates + rows), dim3(kCacheThreads), 0, st, cache_view(s), start, seq_len,
                       (T*)k, (T*)v, c, T_, zero_others, gates);
  });
  return hipGetLastError();
}

}  // namespace fox

// Attention of new tokens over the paged cache (Eq. fot-weight for the last positions of a
// sequence): n tokens of each sequence, in the cache already, attend to every token before
// them and, among the new ones, to their ancestors and themselves (a tree of drafts; a chain
// without `parent`; one decode step with n = 1).  Grouped heads: query head h reads key head
// h / G, G = H / Hkv, with its own forget gate.
//
//     u_ij = log2(e) (s 2^ek_j (q_i . k~_j) + c_i - c_j),   p_ij = 2^(u_ij - m_i),
//     o_i = sum_j p_ij 2^ev_j v~_j / sum_j p_ij,            lse_i = ln 2 (m_i + log2 sum_j p_ij)
//
// with k~, v~ the codes and 2^ek, 2^ev the rows' scales (1 for a bf16 cache): K's scale
// multiplies a score, V's a weight, so the codes go to the matrix cores unscaled (exact in
// bf16) and no element is multiplied on its way.
//
//   * The G n rows of a key head share its keys: rows are r = g n + t, 16 to a tile, RT tiles
//     to a workgroup.  The products are 16x16x32 bf16: S^T = K Q^T (keys on the MFMA's rows,
//     rows r on its columns, so a lane owns one r) and O^T += V^T P^T, whose B operand is the
//     P^T that the first product left in the registers; the key order of the contraction is
//     the accumulator's, given to V alike.
//   * Keys are split over the grid in chunks, and a workgroup's four waves take 32-key tiles
//     in turn, each with its own running maximum and sum: no barrier in the loop.  K comes
//     straight into operand registers (a lane reads 16 bytes of a key); V passes through the
//     wave's LDS by DMA and is read back transposed.  The next tile's loads are in flight
//     while a tile is computed.
//   * A tile of 32 keys is two halves of 16, each inside one page (pages hold 16 tokens or
//     more); a half is addressed through a buffer descriptor that ends where its keys end, so
//     nothing behind the sequence is read, and keys without a page read as zero and are masked.
//   * Scores are exponentiated against the running maximum; only if a lane's sum of a tile
//     exceeds 2^8 is the tile's maximum taken and everything rescaled (bf16 P and the fp32
//     sums absorb the 8 bits).  The row sum adds the unrounded fp32 P, P V takes P rounded to
//     bf16.
#include <algorithm>

#include "fox_internal.h"
#include "kv_cache.h"

namespace fox {

typedef uint32_t u32x4d __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2_t;

constexpr int kCaWaves = 4;
constexpr int kCaThreads = 64 * kCaWaves;
constexpr int kCaTile = 32;                        // keys of a wave's tile
constexpr int kCaRound = kCaWaves * kCaTile;       // keys of one turn of the waves
constexpr float kCaSum = 256.0f;                   // a lane's tile sum above it rescales
constexpr float kCaFloor = -1e30f;                 // the maximum before the first key

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// maximum and sum over the four lanes l % 16 + 16 g
__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Place of 16-byte piece `piece` of key `key` (0..31) in a wave's V tile: a row's pieces are
// exchanged so that the keys and pieces that one transposing read of 32 lanes touches lie in
// different banks.
template <int D, bool F8>
__device__ __forceinline__ int v_swizzle(int key) {
  if constexpr (F8) {
    return D == 128 ? (((key >> 1) & 7) ^ ((key >> 4) << 2)) : (((key >> 2) & 3) ^ ((key >> 4) << 1));
  } else {
    return D == 128 ? 2 * (key & 7) : 2 * ((key >> 1) & 3);
  }
}

// The ancestors of new token `lane` and itself, as bits (pointers doubled).
__device__ __forceinline__ uint64_t ancestors(const int* __restrict__ parent, int nn, int lane) {
  uint64_t bits = 1ull << lane;
  int up = -1;
  if (lane < nn) up = parent ? parent[lane] : lane - 1;
  if (up >= lane) up = -1;
  while (__any(up >= 0)) {
    const int from = up >= 0 ? up : lane;
    const uint32_t lo = __shfl((uint32_t)bits, from), hi = __shfl((uint32_t)(bits >> 32), from);
    const int u = __shfl(up, from);
    if (up >= 0) {
      bits |= ((uint64_t)hi << 32) | lo;
      up = u;
    }
  }
  return bits;
}

template <int D, int RT>
struct CaMerge {
  float o[kCaWaves][16][D + 4];  // one row tile at a time
  float m[kCaWaves][16 * RT], l[kCaWaves][16 * RT];
};

template <int D, bool F8, int RT>
__global__ __launch_bounds__(kCaThreads) void attn_cache_kernel(
    CacheView cv, const bf16* __restrict__ Q, const int* __restrict__ seq_len,
    const int* __restrict__ parent, const int* __restrict__ n_new, bf16* __restrict__ O,
    float* __restrict__ LSE, float* __restrict__ part_o, float* __restrict__ part_ml, int n, int G,
    int n_rowblk, int chunk, int nsplit, float scale_log2) {
  constexpr int ESZ = F8 ? 1 : 2;
  constexpr int CPR = D * ESZ / 16;                    // 16-byte pieces of a row
  constexpr int KL = D * ESZ / 64;                     // 16-byte K loads of a lane per half
  constexpr int NS = D / 32;                           // MFMA steps over the head dimension
  constexpr int VL = kCaTile * D * ESZ / 1024;         // DMA loads of a V tile
  constexpr int NB = D / 16;                           // 16-dim blocks of O^T
  constexpr int VBYTES = kCaTile * D * ESZ;
  union Smem {
    char v[kCaWaves][VBYTES];
    CaMerge<D, RT> merge;
  };
  __shared__ __attribute__((aligned(1024))) Smem sm;

  // row blocks of the same keys follow each other on one XCD
  const int nbase = cv.B * cv.Hkv * nsplit;
  const int base = (int)(blockIdx.x / (8u * n_rowblk)) * 8 + (int)(blockIdx.x % 8u);
  const int rb = (int)(blockIdx.x / 8u) % n_rowblk;
  if (base >= nbase) return;
  const int hk = base % cv.Hkv, b = base / cv.Hkv % cv.B, split = base / cv.Hkv / cv.B;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int cap = (int)cv.capacity();
  const int len = min(max(seq_len[b], 0), cap);
  const int nn = n_new ? max(0, min(n_new[b], n)) : n;
  const int T = min(len + nn, cap);
  const int k0 = split * chunk;
  const int k1 = split == nsplit - 1 ? T : min(T, k0 + chunk);
  if (nn == 0 || (k0 >= T && split > 0)) return;

  // this lane's rows
  int head[RT], tok[RT];
  bool row_ok[RT];       // a row of this call
  float ci[RT];
  uint64_t anc[RT];
  bf16x8 qf[RT][NS];
  const uint64_t bits = k1 > len ? ancestors(parent ? parent + (size_t)b * n : nullptr, nn, lane) : 0;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = (rb * RT + i) * 16 + col;
    const int g = r / n;
    tok[i] = r - g * n;
    row_ok[i] = g < G && tok[i] < nn;
    head[i] = hk * G + (row_ok[i] ? g : 0);
    // a token whose own place is not in the cache has no c and sees nothing
    const int own = row_ok[i] && len + tok[i] < cap ? cv.page_of(b, len + tok[i]) : -1;
    ci[i] = own < 0 ? -INFINITY : cv.c[cv.c_at(own, head[i], cv.slot_of(len + tok[i]))];
    const uint32_t lo = __shfl((uint32_t)bits, tok[i]), hi = __shfl((uint32_t)(bits >> 32), tok[i]);
    anc[i] = ((uint64_t)hi << 32) | lo;
    if (own < 0) row_ok[i] = false;
    const bf16* q = Q + (((size_t)b * cv.H + head[i]) * n + (row_ok[i] ? tok[i] : 0)) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      // the dims in the order in which a lane's 16-byte pieces of K hold them
      const int d0 = F8 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp;
      qf[i][s] = *reinterpret_cast<const bf16x8*>(q + d0);
    }
  }

  f32x4 oacc[RT][NB];
  float m[RT], l[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = kCaFloor;
    l[i] = 0.0f;
#pragma unroll
    for (int db = 0; db < NB; ++db) oacc[i][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  struct Half {       // 16 keys of one page
    u32x4d k[KL];
    f32x4 c[RT];
    uint32_t ke, ve;
  };
  struct Tile {
    Half h[2];
    int valid[2];     // keys of each half that exist
  };
  char* vbuf = sm.v[wave];
  // The page numbers of a tile's halves, looked up one tile before its loads are issued.
  auto lookup = [&](int key0, int (&pg)[2]) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) pg[hf] = cv.page_of(b, key0 + 16 * hf);
  };
  auto issue = [&](int key0, const int (&pg)[2], Tile& t) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = key0 + 16 * hf;
      const int p = __builtin_amdgcn_readfirstlane(pg[hf]);
      const int slot = cv.slot_of(key);
      t.valid[hf] = p < 0 ? 0 : max(0, min(16, T - key));
      const size_t row = cv.kv_row(max(p, 0), hk, slot);
      const uint32_t bytes = (uint32_t)t.valid[hf] * D * ESZ;
      const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char*>(cv.k) + row * (D * ESZ), bytes);
      const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const char*>(cv.v) + row * (D * ESZ), bytes);
#pragma unroll
      for (int i = 0; i < KL; ++i)
        t.h[hf].k[i] = __builtin_bit_cast(
            u32x4d, __builtin_amdgcn_raw_buffer_load_b128(rk, col * D * ESZ + 64 * i + 16 * grp, 0, 0));
#pragma unroll
      for (int i = 0; i < RT; ++i)
        t.h[hf].c[i] = *reinterpret_cast<const f32x4*>(
            cv.c + cv.c_at(max(p, 0), head[i], slot) + 4 * grp);
      if constexpr (F8) {
        t.h[hf].ke = *reinterpret_cast<const uint32_t*>(cv.ke + row + 4 * grp);
        t.h[hf].ve = *reinterpret_cast<const uint32_t*>(cv.ve + row + 4 * grp);
      }
      // V: place s of the tile holds piece (s % CPR) ^ swizzle of key s / CPR
#pragma unroll
      for (int i = 0; i < VL / 2; ++i) {
        const int s = i * 64 + lane, kr = s / CPR;
        const int piece = (s % CPR) ^ v_swizzle<D, F8>(16 * hf + kr);
        dma16(rv, vbuf + (hf * (VL / 2) + i) * 1024, (uint32_t)(kr * D * ESZ + 16 * piece));
      }
    }
  };

  // byte address in the V tile of this lane's transposing read for dims 0..15
  const char* vread[2];
  if constexpr (F8) {
    const int r8 = col >> 1, key = (r8 < 4 ? 0 : 12) + 4 * grp + r8;
    vread[0] = vbuf + key * D + 16 * v_swizzle<D, F8>(key) + 8 * (col & 1);
    vread[1] = vread[0];
  } else {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = 16 * hf + 4 * grp + (col >> 2);
      vread[hf] = vbuf + key * D * 2 + 16 * (v_swizzle<D, F8>(key) ^ ((col >> 1) & 1)) + 8 * (col & 1);
    }
  }
  auto xor_at = [&](const char* p, int x) {
    return (const lds_byte*)(uintptr_t)((uint32_t)(uintptr_t)lds_ptr(p) ^ (uint32_t)x);
  };

  Tile cur, nxt;
  const int first = k0 + wave * kCaTile;
  int pg[2];
  lookup(first, pg);
  if (first < k1) issue(first, pg, cur);
  lookup(first + kCaRound, pg);
  for (int key0 = first; key0 < k1; key0 += kCaRound) {
    wait_all_memory();
    sched_fence();
    // V of this tile to registers; then the next tile may overwrite it
    bf16x8 va[F8 ? 1 : NB];
    i32x2 v8[F8 ? NB : 1];
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      if constexpr (F8) {
        v8[db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_t*)xor_at(vread[0], 16 * db));
      } else {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)xor_at(vread[0], 32 * db));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)xor_at(vread[1], 32 * db));
        va[db] = cat4(lo, hi);
      }
    }
    wait_lds();
    sched_fence();
    if (key0 + kCaRound < k1) issue(key0 + kCaRound, pg, nxt);
    lookup(key0 + 2 * kCaRound, pg);
    sched_fence();

    // S^T of the two halves
    f32x4 s[RT][2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
      for (int i = 0; i < RT; ++i) s[i][hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        bf16x8 ka;
        if constexpr (F8) {
          const u32x4d w = cur.h[hf].k[st >> 1];
          ka = e4m3_operand(w[2 * (st & 1)], w[2 * (st & 1) + 1]);
        } else {
          ka = __builtin_bit_cast(bf16x8, cur.h[hf].k[st]);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][hf] = mfma16(ka, qf[i][st], s[i][hf]);
      }
    }
    const bool plain = cur.valid[0] == 16 && cur.valid[1] == 16 && key0 + kCaTile <= len;
    float ks[2][4], vs[2][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ks[hf][j] = scale_log2;
        vs[hf][j] = 1.0f;
        if constexpr (F8) {
          ks[hf][j] = scale_log2 * e4m3_scale((cur.h[hf].ke >> (8 * j)) & 255u);
          vs[hf][j] = e4m3_scale((cur.h[hf].ve >> (8 * j)) & 255u);
          // keys that do not exist: their scales are whatever lies there
          if (!plain && 4 * grp + j >= cur.valid[hf]) vs[hf][j] = 0.0f;
        }
      }
    // weights of each row tile and O^T += V^T P^T
    bf16x8 pb[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float u[8];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = (ci[i] - cur.h[hf].c[i][j]) * kLog2e + s[i][hf][j] * ks[hf][j];
          if (!plain) {
            const int kk = key0 + 16 * hf + 4 * grp + j - len;
            const bool seen = row_ok[i] && 4 * grp + j < cur.valid[hf] &&
                              (kk < 0 || ((anc[i] >> (kk & 63)) & 1) != 0);
            if (!seen) x = -INFINITY;
          }
          u[4 * hf + j] = x;
        }
      float p[8], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = exp2_fast(u[e] - m[i]);
        sum += p[e];
      }
      if (__any(sum > kCaSum)) {
        float mt = u[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mt = fmaxf(mt, u[e]);
        const float m_new = fmaxf(m[i], group_max(mt));
        const float alpha = exp2_fast(m[i] - m_new);
        m[i] = m_new;
        l[i] *= alpha;
#pragma unroll
        for (int db = 0; db < NB; ++db) oacc[i][db] *= alpha;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = exp2_fast(u[e] - m_new);
          sum += p[e];
        }
      }
      l[i] += sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[i][e] = to_bf16(p[e] * vs[e >> 2][e & 3]);
    }
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      bf16x8 v;
      if constexpr (F8) v = e4m3_operand((uint32_t)v8[db][0], (uint32_t)v8[db][1]);
      else v = va[db];
#pragma unroll
      for (int i = 0; i < RT; ++i) oacc[i][db] = mfma16(v, pb[i], oacc[i][db]);
    }
    cur = nxt;
  }

  // merge the waves
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float lt = group_sum(l[i]);
    if (grp == 0) {
      sm.merge.m[wave][16 * i + col] = m[i];
      sm.merge.l[wave][16 * i + col] = lt;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    float M = kCaFloor;
#pragma unroll
    for (int w = 0; w < kCaWaves; ++w) M = fmaxf(M, sm.merge.m[w][16 * i + col]);
    const float f = exp2_fast(m[i] - M);
#pragma unroll
    for (int db = 0; db < NB; ++db)
      *reinterpret_cast<f32x4*>(&sm.merge.o[wave][col][16 * db + 4 * grp]) = oacc[i][db] * f;
    __syncthreads();
    for (int item = threadIdx.x; item < 16 * (D / 4); item += kCaThreads) {
      const int rr = item / (D / 4), e = item % (D / 4) * 4;
      const int r = (rb * RT + i) * 16 + rr;
      const int g = r / n, t = r - g * n;
      if (g >= G || t >= nn) continue;
      float Mr = kCaFloor, lr = 0.0f;
#pragma unroll
      for (int w = 0; w < kCaWaves; ++w) Mr = fmaxf(Mr, sm.merge.m[w][16 * i + rr]);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kCaWaves; ++w) {
        lr += sm.merge.l[w][16 * i + rr] * exp2_fast(sm.merge.m[w][16 * i + rr] - Mr);
        o += *reinterpret_cast<const f32x4*>(&sm.merge.o[w][rr][e]);
      }
      const size_t R = ((size_t)b * cv.H + hk * G + g) * n + t;
      if (nsplit == 1) {
        const float inv = lr > 0.0f ? 1.0f / lr : 0.0f;  // a row without a key: zeros, -inf
        bf16x4 w4;
#pragma unroll
        for (int j = 0; j < 4; ++j) w4[j] = to_bf16(o[j] * inv);
        *reinterpret_cast<bf16x4*>(O + R * D + e) = w4;
        if (e == 0) LSE[R] = lr > 0.0f ? kLn2 * (Mr + log2f(lr)) : -INFINITY;
      } else {
        const size_t at = (size_t)split * cv.B * cv.H * n + R;
        *reinterpret_cast<f32x4*>(part_o + at * D + e) = o;
        if (e == 0) {
          part_ml[2 * at] = Mr;
          part_ml[2 * at + 1] = lr;
        }
      }
    }
    if (i + 1 < RT) __syncthreads();
  }
}

// The splits of a row joined: D / 4 lanes hold a row's elements, the lane groups of a
// workgroup take every SG-th split and meet in LDS.
template <int D, int SG>
__global__ __launch_bounds__(D / 4 * SG) void attn_cache_join_kernel(
    const float* __restrict__ part_o, const float* __restrict__ part_ml,
    const int* __restrict__ seq_len, const int* __restrict__ n_new, bf16* __restrict__ O,
    float* __restrict__ LSE, int BH, int H, int n, int cap, int chunk, int nsplit) {
  constexpr int LPR = D / 4;
  __shared__ float so[SG][D];
  __shared__ float sml[SG][2];
  const size_t R = blockIdx.x;
  const int t = (int)(R % n), b = (int)(R / n / H);
  const int nn = n_new ? max(0, min(n_new[b], n)) : n;
  if (t >= nn) return;
  const int T = min(min(max(seq_len[b], 0), cap) + nn, cap);
  const int ns = max(1, min(nsplit, (T + chunk - 1) / chunk));
  const size_t stride = (size_t)BH * n;
  const int part = threadIdx.x % LPR, sg = threadIdx.x / LPR;
  float M = kCaFloor, l = 0.0f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = sg; s < ns; s += SG) {
    const size_t at = s * stride + R;
    const float ms = part_ml[2 * at], ls = part_ml[2 * at + 1];
    const f32x4 os = *reinterpret_cast<const f32x4*>(part_o + at * D + 4 * part);
    const float Mn = fmaxf(M, ms);
    const float a = exp2_fast(M - Mn), f = exp2_fast(ms - Mn);
    o = o * a + os * f;
    l = l * a + ls * f;
    M = Mn;
  }
  *reinterpret_cast<f32x4*>(&so[sg][4 * part]) = o;
  if (part == 0) {
    sml[sg][0] = M;
    sml[sg][1] = l;
  }
  __syncthreads();
  if (sg > 0) return;
  for (int g = 1; g < SG; ++g) {
    const float ms = sml[g][0], Mn = fmaxf(M, ms);
    const float a = exp2_fast(M - Mn), f = exp2_fast(ms - Mn);
    o = o * a + *reinterpret_cast<const f32x4*>(&so[g][4 * part]) * f;
    l = l * a + sml[g][1] * f;
    M = Mn;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  bf16x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = to_bf16(o[j] * inv);
  *reinterpret_cast<bf16x4*>(O + R * D + 4 * part) = w;
  if (part == 0) LSE[R] = l > 0.0f ? kLn2 * (M + log2f(l)) : -INFINITY;
}

// ---------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------
struct CaPlan {
  int rt, n_rowblk, chunk, nsplit;
};
static CaPlan ca_plan(const CacheSpec& s, int n, int max_len) {
  CaPlan p;
  const int rows = s.H / s.Hkv * n;
  p.rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.n_rowblk = (rows + 16 * p.rt - 1) / (16 * p.rt);
  const long long base = (long long)s.B * s.Hkv * p.n_rowblk;
  const long long most = std::max(1, (max_len + 2 * kCaRound - 1) / (2 * kCaRound));
  const long long want = std::max<long long>(1, 1024 / base);
  const long long ns = std::min(most, want);
  p.chunk = (int)(((max_len + ns - 1) / ns + kCaRound - 1) / kCaRound * kCaRound);
  p.nsplit = (int)((max_len + p.chunk - 1) / p.chunk);
  return p;
}

size_t attn_cache_workspace_bytes(const CacheSpec& s, int n, int max_len) {
  const CaPlan p = ca_plan(s, n, max_len);
  return p.nsplit == 1 ? 0 : (size_t)p.nsplit * s.B * s.H * n * (s.d + 2) * sizeof(float);
}

hipError_t launch_attn_cache(const CacheSpec& s, const void* q, const int* seq_len,
                             const int* parent, const int* n_new, void* o, float* lse, void* ws,
                             int n, int max_len, float scale, hipStream_t st) {
  const CaPlan p = ca_plan(s, n, max_len);
  const size_t rows = (size_t)s.B * s.H * n;
  float* part_o = static_cast<float*>(ws);
  float* part_ml = part_o + (size_t)p.nsplit * rows * s.d;
  const unsigned nbase = (unsigned)s.B * s.Hkv * p.nsplit;
  const dim3 grid((nbase + 7) / 8 * 8 * (unsigned)p.n_rowblk);
  auto run = [&](auto dc, auto f8, auto rt) {
    hipLaunchKernelGGL((attn_cache_kernel<decltype(dc)::value, decltype(f8)::value, decltype(rt)::value>),
                       grid, dim3(kCaThreads), 0, st, cache_view(s), (const bf16*)q, seq_len, parent,
                       n_new, (bf16*)o, lse, part_o, part_ml, n, s.H / s.Hkv, p.n_rowblk, p.chunk,
                       p.nsplit, scale * kLog2e);
  };
  auto by_rows = [&](auto dc, auto f8) {
    if (p.rt == 1) run(dc, f8, std::integral_constant<int, 1>());
    else if (p.rt == 2) run(dc, f8, std::integral_constant<int, 2>());
    else run(dc, f8, std::integral_constant<int, 4>());
  };
  auto by_format = [&](auto dc) {
    if (s.f8) by_rows(dc, std::true_type());
    else by_rows(dc, std::false_type());
  };
  if (s.d == 128) by_format(std::integral_constant<int, 128>());
  else by_format(std::integral_constant<int, 64>());
  if (p.nsplit > 1) {
    const int cap = (int)std::min<long long>((long long)s.max_pages * s.page, 0x7fffffff);
    if (s.d == 128)
      hipLaunchKernelGGL((attn_cache_join_kernel<128, 8>), dim3((unsigned)rows), dim3(256), 0, st,
                         part_o, part_ml, seq_len, n_new, (bf16*)o, lse, s.B * s.H, s.H, n, cap,
                         p.chunk, p.nsplit);
    else
      hipLaunchKernelGGL((attn_cache_join_kernel<64, 16>), dim3((unsigned)rows), dim3(256), 0, st,
                         part_o, part_ml, seq_len, n_new, (bf16*)o, lse, s.B * s.H, s.H, n, cap,
                         p.chunk, p.nsplit);
  }
  return hipGetLastError();
}

}  // namespace fox

// Attention of new tokens over the paged cache (Eq. fot-weight for the last positions of a
// sequence): n tokens of each sequence, in the cache already, attend to every token before
// them and, among the new ones, to their ancestors and themselves (a tree of drafts; a chain
// without `parent`; one decode step with n = 1).  Grouped heads: query head h reads key head
// h / G, G = H / Hkv, with its own forget gate.
//
//     u_ij = log2(e) (s 2^ek_j (q_i . k~_j) + c_i - c_j),   p_ij = 2^(u_ij - m_i),
//     o_i = sum_j p_ij 2^ev_j v~_j / sum_j p_ij,            lse_i = ln 2 (m_i + log2 sum_j p_ij)
//
// with k~, v~ the codes and 2^ek, 2^ev the rows' scales (1 for a bf16 cache).  A lane holds codes
// of one key, whose scale the conversion to bf16 applies (exact; keys whose values are below
// 2^-117 may lose digits that no score sees).  V's scale multiplies a weight before it is
// rounded to bf16, and its codes go to the matrix cores unscaled: a product below 2^-126 may
// vanish, 2^-29 of the largest weight in a row of 2^-90.  Weights reach 2^8 before a rescale, so
// sums over values above 2^100 may overflow (in a bf16 cache too).
//
//   * The G n rows of a key head share its keys: rows are r = g n + t, 16 to a tile.  Two
//     kernels: up to 16 rows (e4m3: 32 or 64) the four waves of a workgroup split the keys of one
//     row tile; with more rows each wave owns one or two row tiles and the waves share the
//     keys' tiles (attn_cache_rows_kernel).  The products are 16x16x32 bf16: S^T = K Q^T (keys on the MFMA's rows,
//     rows r on its columns, so a lane owns one r) and O^T += V^T P^T, whose B operand is the
//     P^T that the first product left in the registers; the key order of the contraction is
//     the accumulator's, given to V alike.
//   * Keys are split over the grid: all sequences' keys together are cut into about as many
//     equal pieces as workgroups are wanted, each within one sequence, from the lengths on the
//     device (ca_piece), so a batch of ragged lengths loads the part evenly.
//   * Splitting, the waves take 32-key tiles in turn, each with its own running maximum and
//     sum: no barrier in the loop.  V passes through the wave's LDS by DMA and is read back
//     transposed; so does K where a row has 128 bytes or less (whole lines to a request: 245 ->
//     228 us at 64 e4m3 sequences, d = 128), and longer rows, whose tiles would halve the
//     resident workgroups, come straight into operand registers.  A tile's loads are issued
//     as soon as the registers and LDS of the one before are read.
//   * A tile of 32 keys is two halves of 16, each inside one page (pages hold 16 tokens or
//     more); a half is addressed through a buffer descriptor that ends where its keys end, so
//     nothing behind the sequence is read, and keys without a page read as zero and are masked.
//   * Tiles are visited from the newest keys backwards: older ones are the more forgotten, so
//     the first tile's maximum serves nearly all others.
//   * Scores are exponentiated against the running maximum; only if a lane's sum of a tile
//     exceeds 2^8 is the tile's maximum taken and everything rescaled (bf16 P and the fp32
//     sums absorb the 8 bits).  The row sum adds the unrounded fp32 P, P V takes P rounded to
//     bf16.
//
// What bounds it: one token per sequence, the bytes of K and V: 64 e4m3 sequences of 8 to 32
// thousand tokens (H = 16, H_kv = 4, d = 128, pages of 64; 1.44 GB) take 228 us, 6.3 TB/s, where a
// plain copy of this part reaches 4.8 and a streaming read 6.6.  A single short sequence is
// launch and latency: 2047 tokens, H = 12, d = 64 6.8 us and 2.6 to join.  Trees: 16 drafts of 16 bf16
// sequences of 100 to 8 thousand tokens 29 us at 5.5 TB/s (and 6 to join); 64 drafts of four e4m3
// sequences of 3 to 16 thousand, H = 16, H_kv = 2 45 us (and 8 to join): 7.8 vector instructions to
// a matrix instruction (the conversion of the codes, which every wave does for itself, the
// exponentials, the weights' scales), which one after the other would take 63% of its cycles
// (matrix 22%); the rest is the wait for tiles and barriers (23% of the waves' cycles), starts and
// ends: a workgroup has about ten tiles.
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

// Place of a 16-byte piece of K in its row: the 16 keys of a half whose pieces one operand
// read touches lie in different banks.
template <int D, bool F8>
__device__ __forceinline__ int k_swizzle(int key) {
  constexpr int BYTES = D * (F8 ? 1 : 2);
  return BYTES == 256 ? key & 15 : BYTES == 128 ? (key >> 1) & 7 : (key >> 2) & 3;
}

// The ancestors of new token `lane`, whose parent is `up`, and itself, as bits (pointers doubled).
__device__ __forceinline__ uint64_t ancestors(int up, int nn, int lane) {
  const uint32_t bit = 1u << (lane & 31);
  uint64_t bits = lane < 32 ? (uint64_t)bit : (uint64_t)bit << 32;
  if (lane >= nn || up >= lane) up = -1;
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

// What a workgroup takes of the keys: positions k0 .. k1 - 1 of sequence b, the split-th of its
// `count` pieces, whose first is number `first` of all.
struct CaPiece {
  int b, len, nn, T, k0, k1, split, count, first;
};
struct CaSplit {
  int unit;       // keys that a piece's length is a multiple of
  int min_units;  // of a piece
  int target;     // pieces wanted; 0: one of each sequence
};
// Units of a piece at most, for `total` units of all sequences (2^40 of them where 2^16 tables of
// 2^30 tokens share pages): never more than a sequence has, so that the number fits, and with it
// the pieces, of which there are target + B at most.
constexpr int kCaOnePiece = 1 << 30;
__host__ __device__ constexpr int ca_most(long long total, const CaSplit& sp) {
  const long long even = sp.target == 0 ? kCaOnePiece : (total + sp.target - 1) / sp.target;
  const long long most = even > sp.min_units ? even : sp.min_units;
  return most < kCaOnePiece ? (int)most : kCaOnePiece;
}
static_assert(ca_most(1000, CaSplit{64, 8, 4}) == 250 && ca_most(5, CaSplit{64, 8, 4}) == 8);
static_assert(ca_most(1LL << 40, CaSplit{64, 8, 1}) == kCaOnePiece);
static_assert(ca_most((1LL << 32) + 100, CaSplit{64, 8, 1}) == kCaOnePiece);
static_assert(ca_most(1000, CaSplit{64, 8, 0}) == kCaOnePiece);
// Piece number `piece`, found by every wave for itself from the lengths of the sequences: with
// W units of keys in all, a piece has max(min_units, ceil(W / target)) units at most, so that
// there are at most target + B of them whatever the lengths, and a sequence's pieces are
// equal.  False: there are fewer pieces.
__device__ __forceinline__ bool ca_piece(const CacheView& cv, const int* __restrict__ seq_len,
                                         const int* __restrict__ n_new, int n, const CaSplit& sp,
                                         int piece, int lane, CaPiece& out) {
  const int cap = (int)cv.capacity();
  int len = 0, nn = 0;  // of the lane's sequence
  auto units_of = [&](int b) {
    const int at = min(b, cv.B - 1);
    len = min(max(seq_len[at], 0), cap);
    nn = n_new ? max(0, min(n_new[at], n)) : n;
    return b >= cv.B || nn == 0 ? 0 : (min(len + nn, cap) + sp.unit - 1) / sp.unit;
  };
  const int u0 = units_of(lane);
  long long total = 0;
  for (int b0 = 0; b0 < cv.B; b0 += 64) {
    long long u = b0 == 0 ? u0 : units_of(b0 + lane);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) u += __shfl_xor(u, off);
    total += u;
  }
  const int most = ca_most(total, sp);
  int first = 0;
  for (int b0 = 0; b0 < cv.B; b0 += 64) {
    const int u = cv.B <= 64 ? u0 : units_of(b0 + lane), pieces = u / most + (u % most != 0);
    int incl = pieces;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    const uint64_t past = __ballot(first + incl > piece);
    if (past) {
      const int l = __builtin_ctzll(past);
      out.b = b0 + l;
      out.count = __builtin_amdgcn_readlane(pieces, l);
      out.first = first + __builtin_amdgcn_readlane(incl, l) - out.count;
      out.split = piece - out.first;
      out.len = __builtin_amdgcn_readlane(len, l);
      out.nn = __builtin_amdgcn_readlane(nn, l);
      out.T = min(out.len + out.nn, cap);
      const int units = __builtin_amdgcn_readlane(u, l);
      const int per = (units + out.count - 1) / out.count * sp.unit;
      out.k0 = out.split * per;
      out.k1 = min(out.T, out.k0 + per);
      return true;
    }
    first += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Where the parts of split sequences meet: the first piece and the number of pieces of each
// sequence, then O and (maximum, sum) of [piece][head of the key head's group, token] rows.
struct CaParts {
  int2* table;  // [B]
  float* o;
  float* ml;
};

// Operand `st` of the first product (16 keys, dims in the order of ca_dim) from a lane's
// 16-byte pieces of its key.
template <bool F8>
__device__ __forceinline__ bf16x8 k_operand(const u32x4d* w, int st, float scale) {
  if constexpr (F8) return e4m3_operand(w[st >> 1][2 * (st & 1)], w[st >> 1][2 * (st & 1) + 1], scale);
  else return __builtin_bit_cast(bf16x8, w[st]);
}
// first of the eight dims that a lane of group grp holds in operand st
template <bool F8>
__device__ __forceinline__ int ca_dim(int st, int grp) {
  return F8 ? 64 * (st >> 1) + 16 * grp + 8 * (st & 1) : 32 * st + 8 * grp;
}

// The scales 2^ev of a lane's four keys, which multiply their weights.
template <bool F8>
struct CaScales {
  float v[F8 ? 4 : 1];
  __device__ __forceinline__ void set(uint32_t ve) {
    if constexpr (F8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = e4m3_scale((ve >> (8 * j)) & 255u);
    }
  }
  // The scales of keys that do not exist are whatever lies there; their weights are 0.
  __device__ __forceinline__ void clear_from(int valid) {
    if constexpr (F8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = j < valid ? v[j] : 0.0f;
    }
  }
};

// Scores in base 2, less `base`, of a lane's four keys of a half.
__device__ __forceinline__ void ca_scores(float* x, const f32x4& s, const f32x4& c, float ci,
                                          float scale_log2, float base) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    x[j] = __builtin_fmaf(s[j], scale_log2, __builtin_fmaf(ci - c[j], kLog2e, -base));
}
// What the scores of a row are taken relative to: its running maximum, once it has seen a key.
__device__ __forceinline__ float ca_base(float m) { return m == kCaFloor ? 0.0f : m; }

// The mask of a lane's four keys of a half in a tile that holds keys from `valid` on, which do
// not exist, or new tokens (from kk = 0 on), of which only ancestors are seen.  The bit is
// taken from one half of the 64: v_lshrrev_b64 with its shift in the last of 256 registers,
// where the compiler had put it, shifted by something else now and then.
__device__ __forceinline__ void ca_mask(float* u, int valid, int kk0, uint64_t anc) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int kk = kk0 + j;
    const uint32_t half = kk & 32 ? (uint32_t)(anc >> 32) : (uint32_t)anc;
    const int seen = (int)(j < valid) & ((int)(kk < 0) | (int)((half >> (kk & 31)) & 1));
    u[j] = seen ? u[j] : -INFINITY;
  }
}

// The weights of one row's 4 NH scores (x, less ca_base(m)), as operands of the second
// product.  Only if a lane's sum exceeds 2^8, or before the row's first key, the scores'
// maximum is taken and everything rescaled.
template <bool F8, int NB, int NH>
__device__ __forceinline__ void ca_softmax(float* x, const CaScales<F8>* sc, float& m, float& l,
                                           f32x4 (&o)[NB], bf16x8* pb) {
  float p[4 * NH], sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 4 * NH; ++e) {
    p[e] = exp2_fast(x[e]);
    sum += p[e];
  }
  if (__any(sum > kCaSum || m == kCaFloor)) {
    float mt = x[0];
#pragma unroll
    for (int e = 1; e < 4 * NH; ++e) mt = fmaxf(mt, x[e]);
    mt = group_max(mt);
    const bool none = m == kCaFloor;
    // a row that still sees nothing stays at the floor; its weights are zeros
    const float shift = none ? (mt == -INFINITY ? 0.0f : mt) : fmaxf(mt, 0.0f);
    const float alpha = none ? 0.0f : exp2_fast(-shift);
    if (!none || mt != -INFINITY) m = ca_base(m) + shift;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < NB; ++db) o[db] *= alpha;
    sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4 * NH; ++e) {
      p[e] = exp2_fast(x[e] - shift);
      sum += p[e];
    }
  }
  l += sum;
#pragma unroll
  for (int e = 0; e < 4 * NH; ++e) {
    if constexpr (F8) pb[e / 8][e % 8] = to_bf16(p[e] * sc[e / 4].v[e % 4]);
    else pb[e / 8][e % 8] = to_bf16(p[e]);
  }
}

// Of 16 keys that start at slot `slot` of page p: the prefix values of the four whose scores a
// lane gets (c_off: of its head in a page), V's scale exponents of these and K's of the one
// whose codes it holds.
template <bool F8, int RT>
__device__ __forceinline__ void ca_load_c(const CacheView& cv, int p, int hk, int slot,
                                          const uint32_t (&c_off)[RT], int col, int grp,
                                          f32x4* c, uint32_t& ke, uint32_t& ve) {
  const __amdgpu_buffer_rsrc_t rc = uniform_rsrc(
      reinterpret_cast<const char*>(cv.c + cv.c_at(p, 0, 0)), (uint32_t)(cv.H << cv.page_shift) * 4);
#pragma unroll
  for (int i = 0; i < RT; ++i)
    c[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, c_off[i], slot * 4, 0));
  if constexpr (F8) {
    const size_t row = cv.kv_row(p, hk, slot);
    const __amdgpu_buffer_rsrc_t rk = uniform_rsrc(reinterpret_cast<const char*>(cv.ke + row), 16);
    const __amdgpu_buffer_rsrc_t rv = uniform_rsrc(reinterpret_cast<const char*>(cv.ve + row), 16);
    ke = __builtin_amdgcn_raw_buffer_load_b8(rk, col, 0, 0);
    ve = __builtin_amdgcn_raw_buffer_load_b32(rv, 4 * grp, 0, 0);
  }
}

// A lane's rows, one of each row tile of its wave: row r is token r % n of head r / n of the
// key head's group.
template <int D, bool F8, int RT>
struct CaRows {
  int head[RT], tok[RT];
  bool mine[RT];    // a row of this call
  bool ok[RT];      // whose own place is in the cache; any other has no c and sees nothing
  float ci[RT];
  uint64_t anc[RT];
  uint32_t c_off[RT];
  bf16x8 q[RT][D / 32];

  __device__ __forceinline__ void place(const CacheView& cv, const CaPiece& pc, int row0, int hk,
                                        int G, int n, int grp) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = row0 + 16 * i, g = r / n;
      tok[i] = r - g * n;
      mine[i] = g < G && tok[i] < pc.nn;
      head[i] = hk * G + (mine[i] ? g : 0);
      tok[i] = mine[i] ? tok[i] : 0;
      c_off[i] = (uint32_t)((head[i] << cv.page_shift) + 4 * grp) * 4;
    }
  }
  // row of O and LSE
  __device__ __forceinline__ size_t out(int i, int b, int H, int n) const {
    return ((size_t)b * H + head[i]) * n + tok[i];
  }
  // Every load is issued whether its lane needs it or not, so that they wait for each other
  // once and not one by one.
  __device__ __forceinline__ void load(const CacheView& cv, const CaPiece& pc,
                                       const bf16* __restrict__ Q, const int* __restrict__ parent,
                                       int n, int lane, int grp) {
    int up = lane - 1, own[RT];
    if (parent) up = parent[(size_t)pc.b * n + min(lane, n - 1)];
#pragma unroll
    for (int i = 0; i < RT; ++i)
      own[i] = cv.table[(size_t)pc.b * cv.max_pages +
                        min((pc.len + tok[i]) >> cv.page_shift, cv.max_pages - 1)];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
        q[i][s] = *reinterpret_cast<const bf16x8*>(Q + out(i, pc.b, cv.H, n) * D + ca_dim<F8>(s, grp));
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      ok[i] = mine[i] && pc.len + tok[i] < (int)cv.capacity() && cv.page_exists(own[i]);
      ci[i] = cv.c[cv.c_at(ok[i] ? own[i] : 0, head[i], cv.slot_of(pc.len + tok[i]))];
    }
    const uint64_t bits = pc.k1 > pc.len ? ancestors(up, pc.nn, lane) : 0;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const uint32_t lo = __shfl((uint32_t)bits, tok[i]), hi = __shfl((uint32_t)(bits >> 32), tok[i]);
      anc[i] = ((uint64_t)hi << 32) | lo;
      ci[i] = ok[i] ? ci[i] : -INFINITY;
    }
  }
};

template <int D>
struct CaMerge {
  float o[kCaWaves][16][D + 4];
  float m[kCaWaves][16], l[kCaWaves][16];
};

// NT: K and V bypass the caches (read once, and more than they hold).
template <bool NT>
__device__ __forceinline__ void ca_dma16(__amdgpu_buffer_rsrc_t r, void* lds, uint32_t off) {
  if constexpr (NT) dma16_nt(r, lds, off);
  else dma16(r, lds, off);
}

template <int D, bool F8, bool NT>
__global__ __launch_bounds__(kCaThreads) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 3)))
void attn_cache_kernel(
    CacheView cv, const bf16* __restrict__ Q, const int* __restrict__ seq_len,
    const int* __restrict__ parent, const int* __restrict__ n_new, bf16* __restrict__ O,
    float* __restrict__ LSE, CaParts parts, CaSplit sp, int n, int G, int n_rowblk, int n_pieces,
    float scale_log2) {
  constexpr int ESZ = F8 ? 1 : 2;
  constexpr int CPR = D * ESZ / 16;                    // 16-byte pieces of a row
  constexpr int KL = D * ESZ / 64;                     // 16-byte K loads of a lane per half
  constexpr int NS = D / 32;                           // MFMA steps over the head dimension
  constexpr int VL = kCaTile * D * ESZ / 1024;         // DMA loads of a V tile
  constexpr int NB = D / 16;                           // 16-dim blocks of O^T
  constexpr int VBYTES = kCaTile * D * ESZ;
  constexpr bool KLDS = D * ESZ <= 128;                // K through LDS too
  union Smem {
    char v[kCaWaves][(KLDS ? 2 : 1) * VBYTES];  // V, then K
    CaMerge<D> merge;
  };
  __shared__ __attribute__((aligned(1024))) Smem sm;

  // row blocks of the same keys follow each other on one XCD
  const int nbase = cv.Hkv * n_pieces;
  const int base = (int)(blockIdx.x / (8u * n_rowblk)) * 8 + (int)(blockIdx.x % 8u);
  const int rb = (int)(blockIdx.x / 8u) % n_rowblk;
  if (base >= nbase) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hk = base % cv.Hkv;
  CaPiece pc;
  if (!ca_piece(cv, seq_len, n_new, n, sp, base / cv.Hkv, lane, pc)) return;
  const int b = pc.b, len = pc.len, nn = pc.nn, T = pc.T, k0 = pc.k0, k1 = pc.k1;
  const int cap = (int)cv.capacity();
  if (pc.split == 0 && hk == 0 && rb == 0 && threadIdx.x == 0 && parts.table)
    parts.table[b] = make_int2(pc.first, pc.count);
  const int col = lane & 15, grp = lane >> 4;

  CaRows<D, F8, 1> rows;
  rows.place(cv, pc, rb * 16 + col, hk, G, n, grp);
  struct Half {       // 16 keys of one page
    u32x4d k[KLDS ? 1 : KL];  // without KLDS
    f32x4 c;
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
    for (int hf = 0; hf < 2; ++hf) pg[hf] = cv.page_entry(b, key0 + 16 * hf);
  };
  auto issue = [&](int key0, const int (&pg)[2], Tile& t) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = key0 + 16 * hf;
      const bool there = cv.page_exists(pg[hf]) && key < T;
      const int p = __builtin_amdgcn_readfirstlane(there ? pg[hf] : 0);
      const int slot = cv.slot_of(key);
      t.valid[hf] = there ? min(16, T - key) : 0;
      const size_t row = cv.kv_row(p, hk, slot);
      const uint32_t bytes = (uint32_t)t.valid[hf] * D * ESZ;
      const __amdgpu_buffer_rsrc_t rk = uniform_rsrc(static_cast<const char*>(cv.k) + row * (D * ESZ), bytes);
      const __amdgpu_buffer_rsrc_t rv = uniform_rsrc(static_cast<const char*>(cv.v) + row * (D * ESZ), bytes);
      if constexpr (!KLDS) {
#pragma unroll
        for (int i = 0; i < KL; ++i)
          t.h[hf].k[i] = __builtin_bit_cast(
              u32x4d, __builtin_amdgcn_raw_buffer_load_b128(rk, col * D * ESZ + 64 * i + 16 * grp, 0,
                                                             NT ? kNonTemporal : 0));
      }
      ca_load_c<F8, 1>(cv, p, hk, slot, rows.c_off, col, grp, &t.h[hf].c, t.h[hf].ke, t.h[hf].ve);
      // V: place s of the tile holds piece (s % CPR) ^ swizzle of key s / CPR
#pragma unroll
      for (int i = 0; i < VL / 2; ++i) {
        const int s = i * 64 + lane, kr = s / CPR;
        const int piece = (s % CPR) ^ v_swizzle<D, F8>(16 * hf + kr);
        ca_dma16<NT>(rv, vbuf + (hf * (VL / 2) + i) * 1024, (uint32_t)(kr * D * ESZ + 16 * piece));
        if constexpr (KLDS)
          ca_dma16<NT>(rk, vbuf + VBYTES + (hf * (VL / 2) + i) * 1024,
                       (uint32_t)(kr * D * ESZ + 16 * ((s % CPR) ^ k_swizzle<D, F8>(kr))));
      }
    }
  };

  const lds_byte* kat[KL];  // KLDS: this lane's pieces of its key
#pragma unroll
  for (int i = 0; i < KL; ++i)
    kat[i] = lds_ptr(vbuf) + VBYTES + col * D * ESZ + 16 * ((4 * i + grp) ^ k_swizzle<D, F8>(col));
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

  // A tile's registers and LDS are refilled as soon as they have been read, before the second
  // product: half the registers of a second set, so twice the waves, which hide more of the
  // latency than the set did.
  Tile cur;
  const int first = k0 + wave * kCaTile;
  const int last = first < k1 ? first + (k1 - 1 - first) / kCaRound * kCaRound : first - 1;
  int pg[2];
  lookup(last, pg);
  if (first < k1) issue(last, pg, cur);
  lookup(last - kCaRound, pg);
  rows.load(cv, pc, Q, parent, n, lane, grp);
  f32x4 oacc[NB];
  float m = rows.ok[0] ? kCaFloor : 0.0f, l = 0.0f;
#pragma unroll
  for (int db = 0; db < NB; ++db) oacc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int key0 = last; key0 >= first; key0 -= kCaRound) {
    wait_all_memory();
    sched_fence();
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

    // S^T of the two halves
    f32x4 s[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      s[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
      u32x4d kw[KL];
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        if constexpr (KLDS) kw[i] = __builtin_bit_cast(u32x4d, *(const lds_f32x4_t*)(kat[i] + hf * 16 * D * ESZ));
        else kw[i] = cur.h[hf].k[i];
      }
#pragma unroll
      for (int st = 0; st < NS; ++st)
        s[hf] = mfma16(k_operand<F8>(kw, st, e4m3_scale(cur.h[hf].ke)), rows.q[0][st], s[hf]);
    }
    const bool plain = cur.valid[0] == 16 && cur.valid[1] == 16 && key0 + kCaTile <= len;
    bf16x8 pb;
    CaScales<F8> sc[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) sc[hf].set(cur.h[hf].ve);
    if (!plain)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) sc[hf].clear_from(cur.valid[hf] - 4 * grp);
    float x[8];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
      ca_scores(x + 4 * hf, s[hf], cur.h[hf].c, rows.ci[0], scale_log2, ca_base(m));
    if (!plain)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        ca_mask(x + 4 * hf, rows.ok[0] ? cur.valid[hf] - 4 * grp : 0,
                key0 + 16 * hf + 4 * grp - len, rows.anc[0]);
    ca_softmax<F8, NB, 2>(x, sc, m, l, oacc, &pb);
    sched_fence();
    wait_lds();  // V is in registers
    if (key0 > first) issue(key0 - kCaRound, pg, cur);
    lookup(key0 - 2 * kCaRound, pg);
    sched_fence();
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      bf16x8 v;
      if constexpr (F8) v = e4m3_operand((uint32_t)v8[db][0], (uint32_t)v8[db][1], 1.0f);
      else v = va[db];
      oacc[db] = mfma16(v, pb, oacc[db]);
    }
  }

  // merge the waves
  const float lt = group_sum(l);
  __syncthreads();  // the V tiles are done with
  if (grp == 0) {
    sm.merge.m[wave][col] = m;
    sm.merge.l[wave][col] = lt;
  }
  __syncthreads();
  float M = kCaFloor;
#pragma unroll
  for (int w = 0; w < kCaWaves; ++w) M = fmaxf(M, sm.merge.m[w][col]);
  const float f = exp2_fast(m - M);
#pragma unroll
  for (int db = 0; db < NB; ++db)
    *reinterpret_cast<f32x4*>(&sm.merge.o[wave][col][16 * db + 4 * grp]) = oacc[db] * f;
  __syncthreads();
  for (int item = threadIdx.x; item < 16 * (D / 4); item += kCaThreads) {
    const int rr = item / (D / 4), e = item % (D / 4) * 4;
    const int r = rb * 16 + rr, g = r / n, t = r - g * n;
    if (g >= G || t >= nn) continue;
    float Mr = kCaFloor, lr = 0.0f;
#pragma unroll
    for (int w = 0; w < kCaWaves; ++w) Mr = fmaxf(Mr, sm.merge.m[w][rr]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kCaWaves; ++w) {
      lr += sm.merge.l[w][rr] * exp2_fast(sm.merge.m[w][rr] - Mr);
      o += *reinterpret_cast<const f32x4*>(&sm.merge.o[w][rr][e]);
    }
    const size_t R = ((size_t)b * cv.H + hk * G + g) * n + t;
    if (pc.count == 1) {
      const float inv = lr == 0.0f ? 0.0f : 1.0f / lr;  // a row without a key: zeros, -inf
      bf16x4 w4;
#pragma unroll
      for (int j = 0; j < 4; ++j) w4[j] = to_bf16(o[j] * inv);
      *reinterpret_cast<bf16x4*>(O + R * D + e) = w4;
      if (e == 0) LSE[R] = lr == 0.0f ? -INFINITY : kLn2 * (Mr + log2f(lr));
    } else {
      const size_t at = ((size_t)(pc.first + pc.split) * cv.H + hk * G + g) * n + t;
      *reinterpret_cast<f32x4*>(parts.o + at * D + e) = o;
      if (e == 0) {
        parts.ml[2 * at] = Mr;
        parts.ml[2 * at + 1] = lr;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows (trees, large groups): the four waves of a workgroup own RT row tiles each and
// walk the same 64-key tiles, K and V of which pass through LDS once for all of them, moved by
// DMA and double-buffered, wave w moving the w-th 16 keys.  One barrier per tile; a wave's
// rows are its own, so nothing is merged at the end.
// ---------------------------------------------------------------------------
constexpr int kCrTile = 64;

// transposing read of 8-bit elements at a byte address, as ds_read_tr_asm; valid after
// lds_wait8()
template <int OFF>
__device__ __forceinline__ i32x2 ds_read_tr8_asm(uint32_t base) {
  i32x2 r;
  asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(r) : "v"(base), "i"(OFF));
  return r;
}
template <int N, int M>
__device__ __forceinline__ void lds_wait8(i32x2 (&r)[M]) {
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"i"(N));
#pragma unroll
  for (int i = 0; i < M; ++i) asm volatile("" : "+v"(r[i]));
}

template <int D, bool F8>
struct CrSmem {
  char k[2][kCrTile * D * (F8 ? 1 : 2)];
  char v[2][kCrTile * D * (F8 ? 1 : 2)];
};

template <int D, bool F8, int RT, bool NT>
__global__ __launch_bounds__(kCaThreads) __attribute__((amdgpu_waves_per_eu(2)))
void attn_cache_rows_kernel(
    CacheView cv, const bf16* __restrict__ Q, const int* __restrict__ seq_len,
    const int* __restrict__ parent, const int* __restrict__ n_new, bf16* __restrict__ O,
    float* __restrict__ LSE, CaParts parts, CaSplit sp, int n, int G, int n_rowblk, int n_pieces,
    float scale_log2) {
  constexpr int ESZ = F8 ? 1 : 2;
  constexpr int ROW = D * ESZ, CPR = ROW / 16;
  constexpr int KL = ROW / 64;           // 16-byte operand pieces of a lane per half
  constexpr int NS = D / 32, NB = D / 16;
  constexpr int HL = 16 * ROW / 1024;    // DMA loads of a half
  constexpr int TB = kCrTile * ROW;      // bytes of a tile of K or V
  __shared__ __attribute__((aligned(1024))) CrSmem<D, F8> sm;

  const int nbase = cv.Hkv * n_pieces;
  const int base = (int)(blockIdx.x / (8u * n_rowblk)) * 8 + (int)(blockIdx.x % 8u);
  const int rb = (int)(blockIdx.x / 8u) % n_rowblk;
  if (base >= nbase) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hk = base % cv.Hkv;
  CaPiece pc;
  if (!ca_piece(cv, seq_len, n_new, n, sp, base / cv.Hkv, lane, pc)) return;
  const int b = pc.b, len = pc.len, nn = pc.nn, T = pc.T, k0 = pc.k0, k1 = pc.k1;
  const int cap = (int)cv.capacity();
  if (pc.split == 0 && hk == 0 && rb == 0 && threadIdx.x == 0 && parts.table)
    parts.table[b] = make_int2(pc.first, pc.count);
  const int col = lane & 15, grp = lane >> 4;

  CaRows<D, F8, RT> rows;
  rows.place(cv, pc, (rb * kCaWaves + wave) * RT * 16 + col, hk, G, n, grp);
  // K and V of a tile to LDS: a wave moves its own 16 keys.  The lane's source offsets are
  // formed anew for each tile (a few operations; kept, they would be spilled).
  auto issue_kv = [&](int key0, int entry, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    const int key = key0 + 16 * wave;
    const bool there = cv.page_exists(entry) && key < T;
    const size_t row = cv.kv_row(there ? entry : 0, hk, cv.slot_of(key));
    const uint32_t bytes = there ? (uint32_t)min(16, T - key) * ROW : 0u;
    const __amdgpu_buffer_rsrc_t rk = uniform_rsrc(static_cast<const char*>(cv.k) + row * ROW, bytes);
    const __amdgpu_buffer_rsrc_t rv = uniform_rsrc(static_cast<const char*>(cv.v) + row * ROW, bytes);
    int ln = lane;
    asm volatile("" : "+v"(ln));
#pragma unroll
    for (int i = 0; i < HL; ++i) {
      const int sl = i * 64 + ln, kr = sl / CPR, pc = sl % CPR;
      ca_dma16<NT>(rk, sm.k[B] + wave * 16 * ROW + i * 1024,
            (uint32_t)(kr * ROW + 16 * (pc ^ k_swizzle<D, F8>(kr))));
      ca_dma16<NT>(rv, sm.v[B] + wave * 16 * ROW + i * 1024,
            (uint32_t)(kr * ROW + 16 * (pc ^ v_swizzle<D, F8>(16 * (wave & 1) + kr))));
    }
  };
  // what a wave keeps of a tile in registers: the prefix values and scales of its lanes' keys,
  // refilled once the scores have been formed
  struct Tile {
    f32x4 c[4][RT];
    uint32_t ke[4], ve[4];
    int valid[4];
  };
  auto lookup = [&](int key0, int (&pg)[4]) {
#pragma unroll
    for (int hf = 0; hf < 4; ++hf) pg[hf] = cv.page_entry(b, key0 + 16 * hf);
  };
  auto issue_c = [&](int key0, const int (&pg)[4], Tile& t) {
#pragma unroll
    for (int hf = 0; hf < 4; ++hf) {
      const int key = key0 + 16 * hf, slot = cv.slot_of(key);
      const bool there = cv.page_exists(pg[hf]) && key < T;
      const int p = __builtin_amdgcn_readfirstlane(there ? pg[hf] : 0);
      t.valid[hf] = there ? min(16, T - key) : 0;
      ca_load_c<F8, RT>(cv, p, hk, slot, rows.c_off, col, grp, t.c[hf], t.ke[hf], t.ve[hf]);
    }
  };

  // LDS addresses of the operand reads, opaque: the compiler then adds no wait for the tile
  // that is loading into the other buffer
  const lds_byte* kat[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i)
    kat[i] = lds_opaque(lds_ptr(&sm.k[0][0]) + col * ROW + 16 * ((4 * i + grp) ^ k_swizzle<D, F8>(col)));
  uint32_t vat[2][NB];
#pragma unroll
  for (int db = 0; db < NB; ++db) {
    if constexpr (F8) {
      const int r8 = col >> 1, key = (r8 < 4 ? 0 : 12) + 4 * grp + r8;
      vat[0][db] = lds_addr(&sm.v[0][0]) +
                   (uint32_t)(key * ROW + 16 * (db ^ v_swizzle<D, F8>(key)) + 8 * (col & 1));
      vat[1][db] = vat[0][db];
    } else {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int key = 16 * hf + 4 * grp + (col >> 2);
        vat[hf][db] = lds_addr(&sm.v[0][0]) +
                      (uint32_t)(key * ROW + 16 * ((2 * db + ((col >> 1) & 1)) ^ v_swizzle<D, F8>(key)) +
                                 8 * (col & 1));
      }
    }
  }

  Tile t;
  int pg[4];  // the next tile's pages
  const int last = k0 + (k1 - 1 - k0) / kCrTile * kCrTile;  // (a piece has a key)
  lookup(last, pg);
  int own = cv.page_entry(b, last + 16 * wave);
  issue_kv(last, own, std::integral_constant<int, 0>());
  issue_c(last, pg, t);
  lookup(last - kCrTile, pg);
  own = cv.page_entry(b, last - kCrTile + 16 * wave);
  rows.load(cv, pc, Q, parent, n, lane, grp);
  f32x4 oacc[RT][NB];
  float m[RT], l[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = rows.ok[i] ? kCaFloor : 0.0f;
    l[i] = 0.0f;
#pragma unroll
    for (int db = 0; db < NB; ++db) oacc[i][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto body = [&](int key0, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    f32x4 s[RT][4];
#pragma unroll
    for (int hf = 0; hf < 4; ++hf) {
      u32x4d kw[KL];
#pragma unroll
      for (int i = 0; i < KL; ++i)
        kw[i] = __builtin_bit_cast(u32x4d, *(const lds_f32x4_t*)(kat[i] + B * TB + hf * 16 * ROW));
#pragma unroll
      for (int i = 0; i < RT; ++i) s[i][hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 ka = k_operand<F8>(kw, st, e4m3_scale(t.ke[hf]));
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][hf] = mfma16(ka, rows.q[i][st], s[i][hf]);
      }
    }
    const bool plain = key0 + kCrTile <= len && t.valid[0] == 16 && t.valid[1] == 16 &&
                       t.valid[2] == 16 && t.valid[3] == 16;
    CaScales<F8> sc[4];
#pragma unroll
    for (int hf = 0; hf < 4; ++hf) sc[hf].set(t.ve[hf]);
    if (!plain)
#pragma unroll
      for (int hf = 0; hf < 4; ++hf) sc[hf].clear_from(t.valid[hf] - 4 * grp);
    bf16x8 pb[RT][2];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float x[16];
#pragma unroll
      for (int hf = 0; hf < 4; ++hf)
        ca_scores(x + 4 * hf, s[i][hf], t.c[hf][i], rows.ci[i], scale_log2, ca_base(m[i]));
      if (!plain)
#pragma unroll
        for (int hf = 0; hf < 4; ++hf)
          ca_mask(x + 4 * hf, rows.ok[i] ? t.valid[hf] - 4 * grp : 0,
                  key0 + 16 * hf + 4 * grp - len, rows.anc[i]);
      ca_softmax<F8, NB, 4>(x, sc, m[i], l[i], oacc[i], pb[i]);
    }
    sched_fence();
    if (key0 > k0) issue_c(key0 - kCrTile, pg, t);
    lookup(key0 - 2 * kCrTile, pg);
    sched_fence();
    static_for<2>([&](auto pc) {
      constexpr int P = decltype(pc)::value;  // 32 keys
      constexpr int OFF = B * TB + P * 32 * ROW;
      if constexpr (F8) {
        i32x2 w[NB];
#pragma unroll
        for (int db = 0; db < NB; ++db) w[db] = ds_read_tr8_asm<OFF>(vat[0][db]);
        lds_wait8<0>(w);
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const bf16x8 v = e4m3_operand((uint32_t)w[db][0], (uint32_t)w[db][1], 1.0f);
#pragma unroll
          for (int i = 0; i < RT; ++i) oacc[i][db] = mfma16(v, pb[i][P], oacc[i][db]);
        }
      } else {
        bf16x4 w[2 * NB];
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          w[2 * db] = ds_read_tr_asm<OFF>(vat[0][db]);
          w[2 * db + 1] = ds_read_tr_asm<OFF>(vat[1][db]);
        }
        lds_wait<0>(w);
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
          for (int i = 0; i < RT; ++i)
            oacc[i][db] = mfma16(cat4(w[2 * db], w[2 * db + 1]), pb[i][P], oacc[i][db]);
      }
    });
  };

  auto step = [&](int key0, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    wait_all_memory();
    __syncthreads();  // the tile is in LDS and everybody is done with the one before it
    if (key0 > k0) issue_kv(key0 - kCrTile, own, std::integral_constant<int, 1 - B>());
    own = cv.page_entry(b, key0 - 2 * kCrTile + 16 * wave);
    sched_fence();
    body(key0, bufc);
  };
  for (int key0 = last; key0 >= k0; key0 -= 2 * kCrTile) {
    step(key0, std::integral_constant<int, 0>());
    if (key0 > k0) step(key0 - kCrTile, std::integral_constant<int, 1>());
  }

#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float lt = group_sum(l[i]);
    if (!rows.mine[i]) continue;
    const size_t R = rows.out(i, b, cv.H, n);
    if (pc.count == 1) {
      const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;  // a row without a key: zeros, -inf
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        bf16x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = to_bf16(oacc[i][db][j] * inv);
        *reinterpret_cast<bf16x4*>(O + R * D + 16 * db + 4 * grp) = w;
      }
      if (grp == 0) LSE[R] = lt == 0.0f ? -INFINITY : kLn2 * (m[i] + log2f(lt));
    } else {
      // (piece, head, token): R without its sequence
      const size_t at = (size_t)(pc.first + pc.split - b) * cv.H * n + R;
#pragma unroll
      for (int db = 0; db < NB; ++db)
        *reinterpret_cast<f32x4*>(parts.o + at * D + 16 * db + 4 * grp) = oacc[i][db];
      if (grp == 0) {
        parts.ml[2 * at] = m[i];
        parts.ml[2 * at + 1] = lt;
      }
    }
  }
}

// The pieces of a row joined: D / 4 lanes hold a row's elements, the lane groups of a
// workgroup take every SG-th piece and meet in LDS.
template <int D, int SG>
__global__ __launch_bounds__(D / 4 * SG) void attn_cache_join_kernel(
    CaParts parts, const int* __restrict__ n_new, bf16* __restrict__ O, float* __restrict__ LSE,
    int H, int n) {
  constexpr int LPR = D / 4;
  __shared__ float so[SG][D];
  __shared__ float sml[SG][2];
  const size_t R = blockIdx.x;
  const int t = (int)(R % n), b = (int)(R / n / H);
  if (t >= (n_new ? min(n_new[b], n) : n)) return;
  const int2 pieces = parts.table[b];
  if (pieces.y == 1) return;  // written by its only piece
  const size_t stride = (size_t)H * n, row = (size_t)pieces.x * stride + R - (size_t)b * stride;
  const int part = threadIdx.x % LPR, sg = threadIdx.x / LPR;
  float M = kCaFloor, l = 0.0f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = sg; s < pieces.y; s += SG) {
    const size_t at = s * stride + row;
    const float ms = parts.ml[2 * at], ls = parts.ml[2 * at + 1];
    const f32x4 os = *reinterpret_cast<const f32x4*>(parts.o + at * D + 4 * part);
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
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = to_bf16(o[j] * inv);
  *reinterpret_cast<bf16x4*>(O + R * D + 4 * part) = w;
  if (part == 0) LSE[R] = l == 0.0f ? -INFINITY : kLn2 * (M + log2f(l));
}

// ---------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------
// Which kernel.  The one whose waves split the keys starts and ends faster; the one that shares
// tiles reads and converts them once for 64 or 128 rows.  us at 32 sequences of 8000 tokens, H_kv =
// 4, split / shared: bf16, d = 128 4 rows 93.6 / 88.8, 24 rows 132 / 93; d = 64 16 rows 49.1 / 49.4, 24
// rows 55 / 51; e4m3, d = 128 32 rows 71 / 74, 40 rows 87 / 75; d = 64 32 rows 39 / 62, 64 rows 61 / 66;
// a single bf16 sequence of 2000, d = 128, 4 rows 10.6 / 12.0.
// Two row tiles to a wave halve the tiles' reads and conversions but need twice the rows: 128
// rows, d = 128 two / one, 32 sequences of 8000, H_kv = 2 e4m3 71 / 78, bf16 74 / 78, but one of 2000
// with H_kv = 4 19.4 / 15.6 and 18.0 / 14.0, one of 16000 27.1 / 26.0 and 23.7 / 22.0.
constexpr long long kCrTwo = 1 << 17;  // keys of all workgroups from which two row tiles pay
// How many workgroups the keys are split for.  Sharing: as many as are resident, two or
// three to a CU (512 / 768 / 1024 workgroups, 64 rows: e4m3, one row tile 88 / 80 / 85 us; bf16,
// d = 128 99 / 121 / 111; two row tiles 54 / 62 / 61).  Splitting waves: far more, so that sequences
// of different lengths even out (512 / 1024 / 2048 / 4096: 64 sequences of 8 to 32 thousand
// tokens 250 / 228 / 225 / 226 us).
constexpr long long kCaWant = 2048, kCrWant2 = 512, kCrWant3 = 768;
// The least keys of a piece, 256, 512 or 1024, by the keys of all workgroups: small calls want
// short pieces, larger ones fewer to start and to join.  256 / 512 / 1024, H_kv = 4, e4m3, d = 128:
// one sequence of 2000 9.3 / 10.8 / 13.7 us; one of 30000 17.5 / 14.9 / 17.1; 32 of 2000 22.1 / 19.3 /
// 19.0; 128 of 1000 37.4 / 32.4 / 26.3 (not split).  Sharing, 1024 leaves CUs idle where the
// lengths differ: 64 drafts of four sequences of 3 to 16 thousand tokens 51 / 51 / 66.
constexpr long long kCaSome = 80000, kCaMany = 500000;
// Bytes of K and V from which they bypass the caches when one row block of up to 64 rows reads
// them: 1.5 times the 256 MB that the last level holds.  Two row tiles to a wave (65 to 128 rows)
// go through the caches, whatever their size (the other way was not measured).  us with / without:
// e4m3, d = 128, 64 sequences of 20000 (1.3 GB) 213 / 248, 32 of 8000 (262 MB, in the cache from the
// call before) 56 / 51; bf16 64 of 20000 425 / 462, 32 of 8000 97 / 106.
constexpr long long kCaBypass = 384LL << 20;

struct CaPlan {
  bool shared;  // the kernel for many rows
  int rt, n_rowblk, n_pieces;
  bool once;  // keys bypass the caches
  CaSplit split;
};
static CaPlan ca_plan(const CacheSpec& s, int n, int max_len) {
  CaPlan p;
  const int rows = s.H / s.Hkv * n;
  const long long seqs = (long long)s.B * s.Hkv;
  const bool large = seqs * max_len * 2 * s.d * (s.f8 ? 1 : 2) >= kCaBypass;
  p.shared = rows > (s.f8 ? (s.d == 64 ? 64 : 32) : large && s.d == 128 ? 0 : 16);
  auto blocks = [&](int rt) { return (rows + 64 * rt - 1) / (64 * rt); };
  p.rt = p.shared && rows > 64 && seqs * blocks(2) * max_len >= kCrTwo ? 2 : 1;
  p.n_rowblk = p.shared ? blocks(p.rt) : (rows + 15) / 16;
  const long long all = seqs * p.n_rowblk * max_len;  // keys of all workgroups, at most
  p.once = p.n_rowblk == 1 && p.rt == 1 && large;
  const int least = all < kCaSome ? 256 : all < kCaMany || p.shared ? 512 : 1024;
  const long long want = !p.shared ? kCaWant : p.rt == 2 || (s.d == 128 && !s.f8) ? kCrWant2 : kCrWant3;
  p.split.unit = p.shared ? kCrTile : kCaRound;
  p.split.min_units = (least + p.split.unit - 1) / p.split.unit;
  p.split.target = (int)std::max<long long>(1, want / ((long long)s.Hkv * p.n_rowblk));
  // no more than sequences of max_len make, and none where each is one least piece; longer
  // ones are then cut into larger pieces
  const long long units = ((long long)max_len + p.split.unit - 1) / p.split.unit;
  const long long each = (units + p.split.min_units - 1) / p.split.min_units;
  p.split.target = each == 1 ? 0 : (int)std::min<long long>(p.split.target, each * s.B);
  p.n_pieces = p.split.target + s.B;
  return p;
}
static size_t ca_table_bytes(int B) { return ((size_t)B * sizeof(int2) + 255) & ~(size_t)255; }

size_t attn_cache_workspace_bytes(const CacheSpec& s, int n, int max_len) {
  const CaPlan p = ca_plan(s, n, max_len);
  return p.n_pieces <= s.B ? 0
                           : ca_table_bytes(s.B) +
                                 (size_t)p.n_pieces * s.H * n * (s.d + 2) * sizeof(float);
}

hipError_t launch_attn_cache(const CacheSpec& s, const void* q, const int* seq_len,
                             const int* parent, const int* n_new, void* o, float* lse, void* ws,
                             int n, int max_len, float scale, hipStream_t st) {
  const CaPlan p = ca_plan(s, n, max_len);
  const size_t rows = (size_t)s.B * s.H * n;
  CaParts parts{};
  if (p.n_pieces > s.B) {
    parts.table = static_cast<int2*>(ws);
    parts.o = reinterpret_cast<float*>(static_cast<char*>(ws) + ca_table_bytes(s.B));
    parts.ml = parts.o + (size_t)p.n_pieces * s.H * n * s.d;
  }
  const unsigned nbase = (unsigned)s.Hkv * p.n_pieces;
  const dim3 grid((nbase + 7) / 8 * 8 * (unsigned)p.n_rowblk);
  auto run = [&](auto kernel, auto once) {
    hipLaunchKernelGGL(p.once ? once : kernel, grid, dim3(kCaThreads), 0, st, cache_view(s), (const bf16*)q, seq_len,
                       parent, n_new, (bf16*)o, lse, parts, p.split, n, s.H / s.Hkv, p.n_rowblk,
                       p.n_pieces, scale * kLog2e);
  };
  auto by_rows = [&](auto dc, auto f8) {
    constexpr int D = decltype(dc)::value;
    constexpr bool F8 = decltype(f8)::value;
    // what ca_plan never asks for: large bf16 caches, d = 128, are always shared, and e4m3, d = 64,
    // is shared from 65 rows on, with two row tiles if it is large
    constexpr bool SPLIT_ONCE = F8 || D == 64, SHARE_ONCE = !F8 || D == 128;
    if (p.rt == 2) run(attn_cache_rows_kernel<D, F8, 2, false>, attn_cache_rows_kernel<D, F8, 2, false>);
    else if (p.shared) run(attn_cache_rows_kernel<D, F8, 1, false>,
                           attn_cache_rows_kernel<D, F8, 1, SHARE_ONCE>);
    else run(attn_cache_kernel<D, F8, false>, attn_cache_kernel<D, F8, SPLIT_ONCE>);
  };
  auto by_format = [&](auto dc) {
    if (s.f8) by_rows(dc, std::true_type());
    else by_rows(dc, std::false_type());
  };
  if (s.d == 128) by_format(std::integral_constant<int, 128>());
  else by_format(std::integral_constant<int, 64>());
  if (p.n_pieces > s.B) {
    if (s.d == 128)
      hipLaunchKernelGGL((attn_cache_join_kernel<128, 8>), dim3((unsigned)rows), dim3(256), 0, st,
                         parts, n_new, (bf16*)o, lse, s.H, n);
    else
      hipLaunchKernelGGL((attn_cache_join_kernel<64, 16>), dim3((unsigned)rows), dim3(256), 0, st,
                         parts, n_new, (bf16*)o, lse, s.H, n);
  }
  return hipGetLastError();
}

}  // namespace fox

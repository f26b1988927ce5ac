// Causal Forgetting Attention with grouped heads over packed sequences, bf16: forward
// (appendix, Alg. 1) and both halves of the backward (Alg. 2).
//
// q, o, dO, dq [H, N, d] and k, v, dk, dv [Hkv, N, d] hold the sequences one behind the other;
// query head h reads key head h / G, G = H / Hkv, with its own forget gate.  Per sequence the
// mathematics is that of attn_fwd.hip and attn_bwd.hip, and so are the tiles, the operand
// layouts and the order within a tile: S^T = K Q^T with one query per lane in the forward and
// dQ, the gate bias seeding the accumulator, transposing LDS reads for the second products,
// tiles moved by DMA and double- or triple-buffered.  What differs:
//
//   * A workgroup takes an item of the plan (packed_gates.hip): 128 rows of one sequence, the
//     heaviest first, the heads of an item side by side.  A tile's descriptor ends where the
//     sequence ends, so rows of the next sequence read as zero.
//   * The workgroups of an item's heads are numbered so that an XCD sees few key heads: the G
//     query heads of a key head read the same K and V from its L2.
//   * dK and dV of a key block sum over the G query heads in one workgroup's registers: the
//     loop walks the query tiles of one head after the other (no atomics).  Where the longest
//     such walk would decide the time, the heads are split over workgroups whose fp32 partial
//     sums are added up afterwards (packed_head_split).  dc^k, which belongs to a query head,
//     is written as each head ends.
//   * The row sum l adds the unrounded fp32 P, so that LSE has fp32 errors only, those of its
//     scores: 1e-6 where gates hold on, more where a 128-row block forgets much, since the
//     accumulators start from (c_q0 - c_j) / s and are rounded at that size in each step:
//     2.5e-5, 1.6e-4 and 1.2e-3 for a c that falls by 111, 528 and 3827 over a block (d = 128; at
//     most about 2^-24 (d / 16 + 8) of the fall).  The dQ kernel forms Delta itself from the rows of O and dO that it owns.  The
//     backward forms dS from P rounded to fp16 (2^-12 of it; carried as 2^15 P,
//     which fp16 holds to full precision down to 2^-29) and dc^k adds the unrounded fp32 dS.
//   * c_i shifts a whole softmax row, so dc^q = rowsum(dS) is 0; what it comes out as is the
//     error of Delta, formed from O as rounded to bf16 (or, with o_lo, from O in which only P
//     was: dQ, which takes the Delta that it starts from, is then 2.4e-3 off and not 2.7e-3,
//     where dQ's own rounding is 1.7e-3, for 1% of a training step).  The dQ kernel runs first and adds its
//     row sums (of dS in fp32) to Delta: the dK/dV kernel then sees the Delta of its own P,
//     rows of dS that sum to 0 to fp32 rounding, and d(log f) is the reverse sum of dc^k
//     alone.  bf16 rounding is left in the operands dS and, for dV, P.
//
// Forward and dQ at D = 128 are bound by instruction issue, as the dense kernels: one after the
// other, the instructions would take 81 to 92% of their busy cycles (matrix instructions 53%, and
// the two kinds overlap in part).  dK/dV, at one workgroup per CU, is at 72% and waits 38% of its
// waves' cycles for barriers and LDS.  D = 64 (forward 71, dQ 82, dK/dV 67%) has half the matrix
// work to the same exponentials, short rows that end in masked tiles, and waits 31, 35 and 45%; dK/dV
// has a barrier for every 32 queries.  Prompts of 1001 to 8192 tokens, H = 16, H_kv = 4, D = 128:
// 433 us with prefix and plan (12), 1.07 PFLOP/s of a large library product's 1.36.  Three of 1500 to
// 8191: forward 389, dQ 565, dK/dV 831 us (980, 1010 and 915 TFLOP/s).  Twelve of 64 to 2048, H = 12,
// D = 64: 51, 73 and 97 us (540, 570, 575).
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "fox_internal.h"
#include "packed.h"

namespace fox {

constexpr int kPkThreads = 256;
constexpr int kPkWaves = 4;
constexpr int kPkBM = 32 * kPkWaves;  // query rows of a workgroup
constexpr int kPkBN = 64;             // keys of a tile
static_assert(kPkBM == kPackedBlock, "a workgroup takes one item");
constexpr float kPkRescaleSum = 256.0f;  // a lane's tile sum of P above it rescales

// the item and head of this workgroup; false: nothing to do
struct PackedPlace {
  int len, block, hk, head;
  size_t row, kv_row;  // of the sequence's first row in [H, N] and [Hkv, N]
};
__device__ __forceinline__ bool packed_place(const PackedItem* __restrict__ plan, int bid, int H,
                                             int Hkv, int N, PackedPlace& p) {
  const PackedItem it = packed_item(plan, bid / H, N);
  p.len = it.len;
  p.block = it.block;
  p.head = packed_head(bid % H, Hkv, H / Hkv);
  p.hk = p.head / (H / Hkv);
  p.row = (size_t)p.head * N + it.start;
  p.kv_row = (size_t)p.hk * N + it.start;
  return it.len > 0;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <int D, int KS>
struct alignas(256) PkFwdSmem {
  bf16 k[2][kPkBN * D];
  bf16 v[2][kPkBN * D];
  float c[2][kPkBN];
  float stat[KS > 1 ? kPkWaves : 1][2][64];  // m and l of each lane (split)
  uint32_t arrived;                          // waves of the group that reached its next tile
};

// KS groups of four waves: group g visits key tiles t_last - g, - KS, .. with its own tile
// buffers and barrier, and the groups' O, l and m merge in LDS.
template <int D, int KS>
__global__ __launch_bounds__(kPkThreads * KS)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2)))
void packed_fwd_kernel(const bf16* __restrict__ Q, const bf16* __restrict__ K,
                       const bf16* __restrict__ V, const float* __restrict__ C,
                       bf16* __restrict__ O, bf16* __restrict__ Olo, float* __restrict__ LSE,
                       const PackedItem* __restrict__ plan, int H, int Hkv, int N,
                       float scale_log2) {
  constexpr int TILE = kPkBN * D;
  constexpr int NDMA = TILE * 2 / 1024 / kPkWaves;
  __shared__ __attribute__((aligned(256))) PkFwdSmem<D, KS> smem[KS];

  PackedPlace at;
  if (!packed_place(plan, KS == 1 ? paired_block() : (int)blockIdx.x, H, Hkv, N, at)) return;
  const int L = at.len, q0 = at.block * kPkBM;
  const int tid = threadIdx.x, lane = tid & 63, wave = (tid >> 6) % kPkWaves;
  const int grp = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid / kPkThreads);
  PkFwdSmem<D, KS>& sm = smem[grp];
  const int h = lane >> 5, col = lane & 31;
  const float* c = C + at.row;
  const int qw0 = q0 + wave * 32;
  const int qi = qw0 + col;
  const bool q_valid = qi < L;
  const uint32_t bytes = (uint32_t)L * D * 2;
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(K + at.kv_row * D, bytes);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(V + at.kv_row * D, bytes);

  const uint32_t dma_off = tile_dma_offset<D, kPkWaves>(wave, lane);
  int koff[D / 16];
  tile_row_offsets<D>(koff, col, h);
  int voff[2][D / 32];
  tile_tr_offsets<D>(voff, lane);
  uint32_t vaddr[2][D / 32];
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) vaddr[k2][db] = lds_addr(&sm.v[0][0]) + 2 * voff[k2][db];

  bf16x8 qf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    if (q_valid) {
      qf[s] = *reinterpret_cast<const bf16x8*>(Q + (at.row + qi) * D + 16 * s + 8 * h);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[s][e] = to_bf16(0.0f);
    }
  }
  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.0f;
  float m_used = -INFINITY, l_run = 0.0f;
  const float inv_scale = kLog2e / scale_log2;  // 1 / s

  const int kend = min(L, q0 + kPkBM);
  const int t_last = (kend + kPkBN - 1) / kPkBN - 1;
  const int t_diag = qw0 / kPkBN;  // tile holding this wave's diagonal

  // wave 0 stages the key terms (c_q0 - c_j) / s of the next tile, loaded with the tile's DMA
  // and converted after the tile body (a wait for them would wait for the DMA)
  const float c_q0 = c[q0];
  float craw = 0.0f;
  int ckey = 0;
  auto issue_tile = [&](int kt, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    const uint32_t base = (uint32_t)kt * kPkBN * D * 2;
#pragma unroll
    for (int i = 0; i < NDMA; ++i) {
      const int wslot = (i * kPkWaves + wave) * 512;
      const uint32_t off = dma_off + uniform_u32(base + i * tile_dma_stride<kPkWaves>());
      dma16(rk, &sm.k[B][wslot], off);
      dma16(rv, &sm.v[B][wslot], off);
    }
    if (wave == 0) {
      ckey = kt * kPkBN + lane;
      if (ckey < L) craw = c[ckey];
    }
  };
  auto store_c = [&](auto bufc) {
    constexpr int B = decltype(bufc)::value;
    if (wave == 0) sm.c[B][lane] = (ckey < L ? c_q0 - craw : -INFINITY) * inv_scale;
  };
  auto max32 = [&](const float* u) {
    float mt = u[0];
#pragma unroll
    for (int r = 1; r < 32; ++r) mt = fmaxf(mt, u[r]);
    return wave_max_pair(mt);
  };
  // 32 keys of a staged tile: S^T, seeded with the keys' terms
  auto scores = [&](const bf16* kt_, const float* ct_, f32x16& acc) {
    bf16x8 ka[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) ka[s] = *reinterpret_cast<const bf16x8*>(kt_ + koff[s]);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 ck4 = *reinterpret_cast<const f32x4*>(ct_ + 8 * g + 4 * h);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) acc[4 * g + jj] = ck4[jj];
    }
    sched_fence();
#pragma unroll
    for (int s = 0; s < D / 16; ++s) acc = mfma32(ka[s], qf[s], acc);
  };
  // the same with the causal mask, in base 2
  auto masked_scores = [&](const bf16* kt_, const float* ct_, int key0, float* u) {
    f32x16 acc;
    scores(kt_, ct_, acc);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = acc[r] * scale_log2;
      if (key0 + mfma_row(r, h) > qi) x = -INFINITY;
      u[r] = x;
    }
  };

  auto tile_body = [&](int j, auto bufc, auto masked) {
    constexpr int B = decltype(bufc)::value;
    constexpr bool MASK = decltype(masked)::value;
    const bf16* kt_ = sm.k[B];
    const float* ct_ = sm.c[B];
    float u[32];
    bf16x8 pb[4];
    float psum = 0.0f;
    auto exponentiate = [&](int first, int last) {
#pragma unroll
      for (int cc = first; cc < last; ++cc) {
        float pv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pv[i] = exp2_fast(u[8 * cc + i]);
          psum += pv[i];
        }
        pb[cc] = pack8(pv);
      }
    };
    if constexpr (!MASK) {
      // the scale, exponentials and row sums of keys 0..31 are scheduled between the MFMAs of
      // keys 32..63
      f32x16 acc0, acc1;
      scores(kt_, ct_, acc0);
      bf16x8 ka1[D / 16];
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        ka1[s] = *reinterpret_cast<const bf16x8*>(kt_ + 32 * D + koff[s]);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 ck4 = *reinterpret_cast<const f32x4*>(ct_ + 32 + 8 * g + 4 * h);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) acc1[4 * g + jj] = ck4[jj];
      }
      sched_fence();
#pragma unroll
      for (int r = 0; r < 16; ++r) u[r] = acc0[r] * scale_log2 - m_used;
      exponentiate(0, 2);
#pragma unroll
      for (int s = 0; s < D / 16; ++s) acc1 = mfma32(ka1[s], qf[s], acc1);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
      }
      sched_fence();
#pragma unroll
      for (int r = 0; r < 16; ++r) u[16 + r] = acc1[r] * scale_log2 - m_used;
      exponentiate(2, 4);
      // only if some score exceeds the reference by more than 8 (the lane's sum then exceeds
      // 2^8) is the tile maximum taken
      if (__any(q_valid && psum > kPkRescaleSum)) {
        const float shift = fmaxf(max32(u), 0.0f);
        const float alpha = exp2_fast(-shift);
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) oacc[db] *= alpha;
#pragma unroll
        for (int r = 0; r < 32; ++r) u[r] -= shift;
        m_used += shift;
        psum = 0.0f;
        exponentiate(0, 4);
      }
    } else {
      // the diagonal tile, the first one a wave visits: its row maximum is the reference
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        masked_scores(kt_ + kb * 32 * D, ct_ + kb * 32, j * kPkBN + kb * 32, u + 16 * kb);
      m_used = max32(u);
#pragma unroll
      for (int r = 0; r < 32; ++r) u[r] -= m_used;
      exponentiate(0, 4);
    }
    l_run += psum;
    // O^T += V^T P^T over the four 16-key chunks, the next chunk's operands in flight
    constexpr int NR = 2 * (D / 32);
    bf16x4 tv[2][NR];
    auto read_v = [&](auto cc, bf16x4 (&t)[NR]) {
      constexpr int CH = decltype(cc)::value;
      static_for<D / 32>([&](auto dbc) {
        constexpr int DB = decltype(dbc)::value;
        t[2 * DB] = ds_read_tr_asm<(B * TILE + CH * 16 * D) * 2>(vaddr[0][DB]);
        t[2 * DB + 1] = ds_read_tr_asm<(B * TILE + CH * 16 * D) * 2>(vaddr[1][DB]);
      });
    };
    read_v(std::integral_constant<int, 0>(), tv[0]);
    static_for<4>([&](auto cc) {
      constexpr int CH = decltype(cc)::value;
      if constexpr (CH + 1 < 4) {
        read_v(std::integral_constant<int, CH + 1>(), tv[(CH + 1) % 2]);
        lds_wait<NR>(tv[CH % 2]);
      } else {
        lds_wait<0>(tv[CH % 2]);
      }
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        oacc[db] = mfma32(cat4(tv[CH % 2][2 * db], tv[CH % 2][2 * db + 1]), pb[CH], oacc[db]);
    });
  };

  uint32_t arrivals = 0;
  auto tile_ready = [&]() {
    wait_all_memory();
    if constexpr (KS == 1) __syncthreads();
    else group_sync(&smem[grp].arrived, arrivals += kPkWaves);
  };
  const int j0 = t_last - grp;
  auto step = [&](int j, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    if (KS == 1 || j != j0) tile_ready();  // split, the first tile is awaited below
    if (j >= KS) issue_tile(j - KS, std::integral_constant<int, 1 - B>());
    if (j == t_diag) tile_body(j, bufc, std::true_type());
    else if (j < t_diag) tile_body(j, bufc, std::false_type());
    if (j >= KS) store_c(std::integral_constant<int, 1 - B>());
  };

  if (KS == 1 || j0 >= 0) {
    issue_tile(j0, std::integral_constant<int, 0>());
    store_c(std::integral_constant<int, 0>());
  }
  if constexpr (KS > 1) {
    if (tid < KS) smem[tid].arrived = 0;
    wait_all_memory();
    __syncthreads();  // every group's first tile is in LDS
    // a wave whose diagonal tile is another group's takes its row maximum too, so that every
    // group works from one reference
    if (j0 >= 0 && j0 != t_diag && t_diag <= t_last) {
      const PkFwdSmem<D, KS>& sd = smem[t_last - t_diag];
      float u[32];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        masked_scores(sd.k[0] + kb * 32 * D, sd.c[0] + kb * 32, t_diag * kPkBN + kb * 32,
                      u + 16 * kb);
      m_used = max32(u);
    }
    __syncthreads();  // the groups go on by themselves
  }
  for (int j = j0; j >= 0; j -= 2 * KS) {
    step(j, std::integral_constant<int, 0>());
    if (j >= KS) step(j - KS, std::integral_constant<int, 1>());
  }

  if constexpr (KS > 1) {
    __syncthreads();
    f32x4* part = reinterpret_cast<f32x4*>(&sm.k[0][0]) + wave * (D / 8) * 64 + lane;
    float* stat = &smem[grp].stat[wave][0][lane];
    if (grp > 0) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          part[(4 * db + g) * 64] = f32x4{oacc[db][4 * g], oacc[db][4 * g + 1],
                                          oacc[db][4 * g + 2], oacc[db][4 * g + 3]};
      stat[0] = m_used;
      stat[64] = l_run;
    }
    __syncthreads();
    if (grp > 0) return;
    float M = m_used;
#pragma unroll
    for (int k = 1; k < KS; ++k) M = fmaxf(M, smem[k].stat[wave][0][lane]);
    const float f0 = exp2_fast(m_used - M);
    m_used = M;
    l_run *= f0;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) oacc[db] *= f0;
#pragma unroll
    for (int k = 1; k < KS; ++k) {
      const float f = exp2_fast(smem[k].stat[wave][0][lane] - M);
      l_run += f * smem[k].stat[wave][1][lane];
      const f32x4* pk = reinterpret_cast<const f32x4*>(&smem[k].k[0][0]) + wave * (D / 8) * 64 + lane;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = pk[(4 * db + g) * 64];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) oacc[db][4 * g + jj] += f * v[jj];
        }
    }
  }

  const float l_tot = wave_sum_pair(l_run);
  if (q_valid) {
    const float inv = 1.0f / l_tot;
    const size_t row = (at.row + qi) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const size_t e = row + db * 32 + 8 * g + 4 * h;
        bf16x4 w, lo;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const float x = oacc[db][4 * g + jj] * inv;
          w[jj] = to_bf16(x);
          lo[jj] = to_bf16(x - to_f32(w[jj]));
        }
        *reinterpret_cast<bf16x4*>(O + e) = w;
        if (Olo) *reinterpret_cast<bf16x4*>(Olo + e) = lo;
      }
    if (h == 0) LSE[at.row + qi] = (c[qi] - c_q0) + kLn2 * (m_used + log2f(l_tot));
  }
}

// ---------------------------------------------------------------------------
// dQ, and Delta from dc^q
// ---------------------------------------------------------------------------
// Both backward kernels form P from the same expression, so that its roundings agree: the
// bias is relative to c at the start of the key's aligned block of kPkRef keys.
constexpr int kPkRef = 128;
// P is carried as 2^15 P (see above): the exponent takes the 15, the results the inverse.
constexpr float kPkLift = 15.0f, kPkUnlift = 1.0f / 32768.0f;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) f16x8 lds_f16x8_t;

// Round two floats to fp16 and back as one packed pair.
__device__ __forceinline__ void round_f16_pair(float& a, float& b) {
  f16x2 v = {(_Float16)a, (_Float16)b};
  uint32_t w = __builtin_bit_cast(uint32_t, v);
  asm volatile("" : "+v"(w));
  v = __builtin_bit_cast(f16x2, w);
  a = (float)v[0];
  b = (float)v[1];
}

template <int D, int KS>
struct alignas(256) PkDqSmem {
  bf16 k[2][kPkBN * D];
  bf16 v[2][kPkBN * D];
  float c[2][kPkBN];
  float cref[2];
  float dc[KS > 1 ? kPkWaves : 1][64];
  uint32_t arrived;
};

template <int D>
constexpr int kPkDqGroups = D == 64 ? 3 : 2;

template <int D, int KS>
__global__ __launch_bounds__(kPkThreads * KS)
__attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2)))
void packed_dq_kernel(const bf16* __restrict__ Q, const bf16* __restrict__ K,
                      const bf16* __restrict__ V, const float* __restrict__ C,
                      const float* __restrict__ LSE, const bf16* __restrict__ dO,
                      const bf16* __restrict__ O, const bf16* __restrict__ Olo,
                      float* __restrict__ delta, bf16* __restrict__ dQ, const PackedItem* __restrict__ plan, int H, int Hkv,
                      int N, float scale, float scale_log2) {
  constexpr int TILE = kPkBN * D;
  constexpr int NDMA = TILE * 2 / 1024 / kPkWaves;
  __shared__ __attribute__((aligned(256))) PkDqSmem<D, KS> smem[KS];

  PackedPlace at;
  if (!packed_place(plan, KS == 1 ? paired_block() : (int)blockIdx.x, H, Hkv, N, at)) return;
  const int L = at.len, q0 = at.block * kPkBM;
  const int tid = threadIdx.x, lane = tid & 63, wave = (tid >> 6) % kPkWaves;
  const int grp = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid / kPkThreads);
  PkDqSmem<D, KS>& sm = smem[grp];
  const int h = lane >> 5, col = lane & 31;
  const float* c = C + at.row;
  const int qw0 = q0 + wave * 32;
  const int qi = qw0 + col;
  const bool q_valid = qi < L;
  const uint32_t bytes = (uint32_t)L * D * 2;
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(K + at.kv_row * D, bytes);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(V + at.kv_row * D, bytes);
  const uint32_t dma_off = tile_dma_offset<D, kPkWaves>(wave, lane);
  int roff[D / 16];
  tile_row_offsets<D>(roff, col, h);
  int toff[2][D / 32];
  tile_tr_offsets<D>(toff, lane);

  bf16x8 qf[D / 16], dof[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    if (q_valid) {
      qf[s] = *reinterpret_cast<const bf16x8*>(Q + (at.row + qi) * D + 16 * s + 8 * h);
      dof[s] = *reinterpret_cast<const bf16x8*>(dO + (at.row + qi) * D + 16 * s + 8 * h);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qf[s][e] = to_bf16(0.0f);
        dof[s][e] = to_bf16(0.0f);
      }
    }
  }
  const float cq = q_valid ? c[qi] : 0.0f;
  const float lse_q = q_valid ? LSE[at.row + qi] : 0.0f;
  // Delta_i = dO_i . O_i: a lane holds half of its row's dims, in the pieces of its operands
  float dlt = 0.0f;
  auto add_rows = [&](const bf16* x) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const bf16x8 ov = *reinterpret_cast<const bf16x8*>(x + (at.row + qi) * D + 16 * s + 8 * h);
#pragma unroll
      for (int e = 0; e < 8; ++e) dlt = __builtin_fmaf(to_f32(ov[e]), to_f32(dof[s][e]), dlt);
    }
  };
  if (q_valid) {
    add_rows(O);
    if (Olo) add_rows(Olo);
  }
  dlt = wave_sum_pair(dlt);

  f32x16 dqacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dqacc[db][r] = 0.0f;
  float dcq_part = 0.0f;

  const int kend = min(L, q0 + kPkBM);
  const int t_last = (kend + kPkBN - 1) / kPkBN - 1;
  const int t_diag = qw0 / kPkBN;
  const float inv_scale = 1.0f / scale;
  // wave 0 loads the next tile's prefix values before its share of the tile's DMA and turns
  // them into LDS row terms after the current tile's body
  float craw = 0.0f, crefreg = 0.0f;
  auto issue_tile = [&](int kt, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    const uint32_t base = (uint32_t)kt * kPkBN * D * 2;
    if (wave == 0) {
      const int key = kt * kPkBN + lane;
      crefreg = c[kt * kPkBN / kPkRef * kPkRef];
      craw = key < L ? c[key] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NDMA; ++i) {
      const int wslot = (i * kPkWaves + wave) * 512;
      const uint32_t off = dma_off + uniform_u32(base + i * tile_dma_stride<kPkWaves>());
      dma16(rk, &sm.k[B][wslot], off);
      dma16(rv, &sm.v[B][wslot], off);
    }
  };
  auto store_c = [&](int kt, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    if (wave == 0) {
      sm.c[B][lane] =
          kt * kPkBN + lane < L ? __builtin_fmaf(craw - crefreg, kLog2e, -kPkLift) : INFINITY;
      if (lane == 0) sm.cref[B] = crefreg;
    }
  };

  // LDS operand addresses: a few opaque per-lane registers plus immediates
  constexpr int kVOff = 2 * 2 * TILE;
  typedef PkDqSmem<D, KS> Smem;
  static_assert(offsetof(Smem, v) - offsetof(Smem, k) == (size_t)kVOff,
                "V tiles follow the K tiles");
  const lds_byte* ka_at[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) ka_at[s] = lds_opaque(lds_ptr(&sm.k[0][0]) + 2 * roff[s]);
  uint32_t taddr[2][D / 32];
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      taddr[k2][db] = (uint32_t)(uintptr_t)lds_opaque(lds_ptr(&sm.k[0][0]) + 2 * toff[k2][db]);
  const lds_byte* c_at = lds_opaque(lds_ptr(&sm.c[0][4 * h]));
  const lds_byte* cref_at = lds_opaque(lds_ptr(&sm.cref[0]));

  auto tile_body = [&](int j, auto bufc, auto masked) {
    constexpr int B = decltype(bufc)::value;
    constexpr bool MASK = decltype(masked)::value;
    const int key0 = j * kPkBN;
    const float dref = cq - *(const lds_f32_t*)(cref_at + 4 * B);
    const float bq = (q_valid ? dref - lse_q : -INFINITY) * inv_scale;
    static_for<2>([&](auto kbc) {
      constexpr int kb = decltype(kbc)::value;
      f32x16 sacc, pacc;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sacc[r] = bq;
        pacc[r] = 0.0f;
      }
      {
        bf16x8 ka[D / 16];
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
          ka[s] = *(const lds_bf16x8_t*)(ka_at[s] + 2 * (B * TILE + kb * 32 * D));
        sched_fence();
#pragma unroll
        for (int s = 0; s < D / 16; ++s) sacc = mfma32(ka[s], qf[s], sacc);
      }
      {
        bf16x8 va[D / 16];
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
          va[s] = *(const lds_bf16x8_t*)(ka_at[s] + kVOff + 2 * (B * TILE + kb * 32 * D));
        sched_fence();
#pragma unroll
        for (int s = 0; s < D / 16; ++s) pacc = mfma32(va[s], dof[s], pacc);
      }
      float pv[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 ck4 = *(const lds_f32x4_t*)(c_at + 4 * (B * kPkBN + kb * 32 + 8 * g));
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float p = exp2_fast(sacc[4 * g + jj] * scale_log2 - ck4[jj]);
          if (MASK && key0 + kb * 32 + 8 * g + 4 * h + jj > qi) p = 0.0f;
          pv[4 * g + jj] = p;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; r += 2) round_f16_pair(pv[r], pv[r + 1]);
      float dsv[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dsv[r] = pv[r] * (pacc[r] - dlt);
        dcq_part += dsv[r];
      }
      static_for<2>([&](auto cc) {
        constexpr int ch = decltype(cc)::value;
        constexpr int OFF = 2 * (B * TILE + (2 * kb + ch) * 16 * D);
        const bf16x8 dsb = pack8(&dsv[8 * ch]);
        bf16x4 t[2 * (D / 32)];
        static_for<D / 32>([&](auto dbc) {
          constexpr int db = decltype(dbc)::value;
          t[2 * db] = ds_read_tr_asm<OFF>(taddr[0][db]);
          t[2 * db + 1] = ds_read_tr_asm<OFF>(taddr[1][db]);
        });
        lds_wait<0>(t);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
          dqacc[db] = mfma32(cat4(t[2 * db], t[2 * db + 1]), dsb, dqacc[db]);
      });
    });
  };

  uint32_t arrivals = 0;
  auto step = [&](int j, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    wait_all_memory();
    if constexpr (KS == 1) __syncthreads();
    else group_sync(&smem[grp].arrived, arrivals += kPkWaves);
    if (j >= KS) issue_tile(j - KS, std::integral_constant<int, 1 - B>());
    if (j == t_diag) tile_body(j, bufc, std::true_type());
    else if (j < t_diag) tile_body(j, bufc, std::false_type());
    if (j >= KS) store_c(j - KS, std::integral_constant<int, 1 - B>());
  };
  const int j0 = t_last - grp;
  if constexpr (KS > 1) {
    if (tid < KS) smem[tid].arrived = 0;
    __syncthreads();
  }
  if (KS == 1 || j0 >= 0) {
    issue_tile(j0, std::integral_constant<int, 0>());
    store_c(j0, std::integral_constant<int, 0>());
  }
  for (int j = j0; j >= 0; j -= 2 * KS) {
    step(j, std::integral_constant<int, 0>());
    if (j >= KS) step(j - KS, std::integral_constant<int, 1>());
  }

  if constexpr (KS > 1) {
    __syncthreads();
    if (grp > 0) {
      f32x4* part = reinterpret_cast<f32x4*>(&sm.k[0][0]) + wave * (D / 8) * 64 + lane;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          part[(4 * db + g) * 64] = f32x4{dqacc[db][4 * g], dqacc[db][4 * g + 1],
                                          dqacc[db][4 * g + 2], dqacc[db][4 * g + 3]};
      smem[grp].dc[wave][lane] = dcq_part;
    }
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int k = 1; k < KS; ++k) {
      const f32x4* part = reinterpret_cast<const f32x4*>(&smem[k].k[0][0]) + wave * (D / 8) * 64 + lane;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = part[(4 * db + g) * 64];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) dqacc[db][4 * g + jj] += v[jj];
        }
      dcq_part += smem[k].dc[wave][lane];
    }
  }

  const float dcq_tot = wave_sum_pair(dcq_part) * kPkUnlift;
  const float f = scale * kPkUnlift;
  if (q_valid) {
    bf16* out = dQ + (at.row + qi) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) w[jj] = to_bf16(dqacc[db][4 * g + jj] * f);
        *reinterpret_cast<bf16x4*>(out + db * 32 + 8 * g + 4 * h) = w;
      }
    if (h == 0) delta[at.row + qi] = dlt + dcq_tot;
  }
}

// ---------------------------------------------------------------------------
// dK, dV and dc^k: eight waves own 128 keys as four pairs of 32.  The P wave of a pair forms
// S and P of query tile t and accumulates dV^T, the G wave, one tile behind, dP and dS and
// accumulates dK^T (attn_bwd.hip).  The steps run over the tiles of the G query heads one
// head after the other: step `it` is tile it % n_tiles of head it / n_tiles.
// ---------------------------------------------------------------------------
constexpr int kPkKvWaves = 8;
constexpr int kPkKvThreads = 64 * kPkKvWaves;
constexpr int kPkPairs = kPkKvWaves / 2;
static_assert(32 * kPkPairs == kPackedBlock && kPkRef == kPackedBlock, "an item's keys");

template <int D, int BM>
struct PkKvSmem {
  bf16 q[3][BM * D];
  bf16 g[3][BM * D];
  f16x8 p[3][kPkPairs][BM / 16][64];
  float bq[3][BM];      // ((c_i - c_ref) - LSE_i) / s of each query row
  float dl[3][BM];      // Delta_i
  float raw[2][3][64];  // c_i, LSE_i, Delta_i as loaded, two tiles ahead
  float ck[2];          // c at the block's first key, of the head of an even and odd turn
};

template <int D, int BM>
__global__ __launch_bounds__(kPkKvThreads) __attribute__((amdgpu_waves_per_eu(BM == 32 ? 4 : 2)))
void packed_dkdv_kernel(const bf16* __restrict__ Q, const bf16* __restrict__ K,
                        const bf16* __restrict__ V, const float* __restrict__ C,
                        const float* __restrict__ LSE, const bf16* __restrict__ dO,
                        const float* __restrict__ delta, bf16* __restrict__ dK,
                        bf16* __restrict__ dV, float* __restrict__ dck, float* __restrict__ part,
                        const PackedItem* __restrict__ plan, int H, int Hkv, int splits, int N,
                        float scale, float scale_log2) {
  constexpr int NQB = BM / 32;
  constexpr int TILE = BM * D;
  constexpr int NDMA = TILE * 2 / 1024 / kPkPairs;
  static_assert(NDMA >= 1 && NDMA * kPkPairs * 1024 == TILE * 2, "the P waves cover a tile");
  __shared__ __attribute__((aligned(16))) PkKvSmem<D, BM> sm;

  const PackedItem item = packed_item(plan, blockIdx.x / (Hkv * splits), N);
  if (item.len <= 0) return;
  // the query heads of this workgroup: group hg of G heads of the key head's
  const int L = item.len, hk = (int)(blockIdx.x % Hkv), hg = (int)(blockIdx.x / Hkv % splits);
  const int G = H / Hkv / splits;
  // the item of a sequence's block m does the work of m + 1 blocks; as keys, that is block
  // n_blocks - 1 - m
  const int k0 = ((L + kPackedBlock - 1) / kPackedBlock - 1 - item.block) * kPackedBlock;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = lane >> 5, col = lane & 31;
  const bool pwave = wave < kPkPairs;
  const int pair = wave % kPkPairs;
  const size_t head0 = ((size_t)hk * splits + hg) * G * N + item.start;
  const size_t kv_row = (size_t)hk * N + item.start;
  const int kw0 = k0 + pair * 32;
  const int kj = kw0 + col;
  const bool k_valid = kj < L;
  const uint32_t bytes = (uint32_t)L * D * 2;
  const uint32_t dma_off = tile_dma_offset<D, kPkPairs>(pair, lane);
  int roff[D / 16];
  tile_row_offsets<D>(roff, col, h);
  int toff[2][D / 32];
  tile_tr_offsets<D>(toff, lane);
  const lds_byte* plain_base = pwave ? lds_ptr(&sm.q[0][0]) : lds_ptr(&sm.g[0][0]);
  const lds_byte* tr_base = pwave ? lds_ptr(&sm.g[0][0]) : lds_ptr(&sm.q[0][0]);
  const lds_byte* pa[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) pa[s] = lds_opaque(plain_base + 2 * roff[s]);
  const lds_byte* p_at = lds_opaque(lds_ptr(&sm.p[0][pair][0][lane]));
  const lds_byte* row_at = lds_opaque(lds_ptr(&sm.bq[0][4 * h]));
  constexpr int kPBuf = kPkPairs * (BM / 16) * 64 * 16;
  constexpr int kDlOff = 3 * BM * 4;
  auto plain_op = [&](int s, int boff) { return *(const lds_bf16x8_t*)(pa[s] + boff); };
  uint32_t taddr[2][D / 32];
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      taddr[k2][db] = (uint32_t)(uintptr_t)lds_opaque(tr_base + 2 * toff[k2][db]);
  constexpr int NR = 2 * (D / 32);
  auto read_tr = [&](auto bufc, auto chc, bf16x4 (&t)[NR]) {
    constexpr int OFF = 2 * (decltype(bufc)::value * TILE + decltype(chc)::value * 16 * D);
    static_for<D / 32>([&](auto dbc) {
      constexpr int DB = decltype(dbc)::value;
      t[2 * DB] = ds_read_tr_asm<OFF>(taddr[0][DB]);
      t[2 * DB + 1] = ds_read_tr_asm<OFF>(taddr[1][DB]);
    });
  };

  // P waves hold K rows, G waves hold V rows
  bf16x8 kvf[D / 16];
  {
    const bf16* src = (pwave ? K : V) + (kv_row + kj) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      if (k_valid) {
        kvf[s] = *reinterpret_cast<const bf16x8*>(src + 16 * s + 8 * h);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) kvf[s][e] = to_bf16(0.0f);
      }
    }
  }
  f32x16 acc[D / 32];  // dV^T (P waves) or dK^T (G waves)
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[db][r] = 0.0f;
  float dck_part = 0.0f;

  const int t_first = k0 / BM;
  const int nt = (L + BM - 1) / BM - t_first;  // query tiles of one head
  const int total = nt * G;
  const int t_diag = kw0 / BM;
  const float inv_scale = 1.0f / scale;

  // (head, tile) of a step, advanced one step at a time
  struct Turn {
    int g, t;
  };
  auto next = [&](Turn x) { return x.t + 1 == nt ? Turn{x.g + 1, 0} : Turn{x.g, x.t + 1}; };
  auto row_of = [&](int g) { return head0 + (size_t)g * N; };

  auto issue_stats = [&](Turn x, int rb) {
    if (wave == 0) {
      const size_t row = row_of(x.g);
      const uint32_t nb = (uint32_t)L * 4, off = ((uint32_t)(t_first + x.t) * BM + lane) * 4;
      dma4(make_rsrc(C + row, nb), &sm.raw[rb][0][0], off);
      dma4(make_rsrc(LSE + row, nb), &sm.raw[rb][1][0], off);
      dma4(make_rsrc(delta + row, nb), &sm.raw[rb][2][0], off);
    }
  };
  // c at k0 of the head that the converted tiles belong to (wave 0), of the head that the P
  // waves work on, and the key's term (c_j - c_k0) log2(e) of that head
  float conv_ck0 = C[row_of(0) + k0];
  float ck2 = k_valid ? __builtin_fmaf(C[row_of(0) + kj] - conv_ck0, kLog2e, -kPkLift) : INFINITY;
  float next_ckj = 0.0f, next_ck0 = 0.0f;
  auto convert_stats = [&](Turn x, int rb, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    if (wave == 0 && lane < BM) {
      const int qq = (t_first + x.t) * BM + lane;
      // (behind the sequence the infinity that the scale, of either sign, turns into -infinity)
      sm.bq[B][lane] = (qq < L ? (sm.raw[rb][0][lane] - conv_ck0) - sm.raw[rb][1][lane] : -INFINITY) *
                       inv_scale;
      sm.dl[B][lane] = qq < L ? sm.raw[rb][2][lane] : 0.0f;
    }
  };
  auto issue_tile = [&](Turn x, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    const uint32_t base = (uint32_t)(t_first + x.t) * BM * D * 2;
    if (pwave) {
      const size_t row = row_of(x.g);
      const __amdgpu_buffer_rsrc_t rq = make_rsrc(Q + row * D, bytes);
      const __amdgpu_buffer_rsrc_t rg = make_rsrc(dO + row * D, bytes);
#pragma unroll
      for (int i = 0; i < NDMA; ++i) {
        const int wslot = (i * kPkPairs + pair) * 512;
        const uint32_t off = dma_off + uniform_u32(base + i * tile_dma_stride<kPkPairs>());
        dma16(rq, &sm.q[B][wslot], off);
        dma16(rg, &sm.g[B][wslot], off);
      }
    }
  };

  // P wave on tile qt held in buffer B
  auto p_tile = [&](int qt, auto bufc, auto masked) {
    constexpr int B = decltype(bufc)::value;
    constexpr bool MASK = decltype(masked)::value;
    const int qs0 = qt * BM;
    static_for<NQB>([&](auto qbc) {
      constexpr int qb = decltype(qbc)::value;
      bf16x8 qa[D / 16];
#pragma unroll
      for (int s = 0; s < D / 16; ++s) qa[s] = plain_op(s, 2 * (B * TILE + qb * 32 * D));
      f32x16 sacc;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 bq4 = *(const lds_f32x4_t*)(row_at + 4 * (B * BM + qb * 32 + 8 * g));
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) sacc[4 * g + jj] = bq4[jj];
      }
#pragma unroll
      for (int s = 0; s < D / 16; ++s) sacc = mfma32(qa[s], kvf[s], sacc);
      bf16x4 tr[NR];
      read_tr(bufc, std::integral_constant<int, 2 * qb>(), tr);
      float pv[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ql = qb * 32 + 8 * g + 4 * h;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float p = exp2_fast(sacc[4 * g + jj] * scale_log2 - ck2);
          if (MASK && kj > qs0 + ql + jj) p = 0.0f;
          pv[4 * g + jj] = p;
        }
      }
      static_for<2>([&](auto cc) {
        constexpr int ch = decltype(cc)::value;
        const bf16x8 pb = pack8(&pv[8 * ch]);
        f16x8 ph;
#pragma unroll
        for (int i = 0; i < 8; ++i) ph[i] = (_Float16)pv[8 * ch + i];
        *(lds_f16x8_t*)(p_at + B * kPBuf + (2 * qb + ch) * 1024) = ph;
        lds_wait<1>(tr);  // the store may stay in flight
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
          acc[db] = mfma32(cat4(tr[2 * db], tr[2 * db + 1]), pb, acc[db]);
        if constexpr (ch == 0) read_tr(bufc, std::integral_constant<int, 2 * qb + 1>(), tr);
      });
    });
  };
  // G wave on the tile held in buffer B
  auto g_tile = [&](auto bufc) {
    constexpr int B = decltype(bufc)::value;
    static_for<NQB>([&](auto qbc) {
      constexpr int qb = decltype(qbc)::value;
      bf16x8 ga[D / 16];
#pragma unroll
      for (int s = 0; s < D / 16; ++s) ga[s] = plain_op(s, 2 * (B * TILE + qb * 32 * D));
      f32x16 pacc;
#pragma unroll
      for (int r = 0; r < 16; ++r) pacc[r] = 0.0f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) pacc = mfma32(ga[s], kvf[s], pacc);
      bf16x4 tr[NR];
      read_tr(bufc, std::integral_constant<int, 2 * qb>(), tr);
      static_for<2>([&](auto cc) {
        constexpr int ch = decltype(cc)::value;
        const f16x8 ph = *(const lds_f16x8_t*)(p_at + B * kPBuf + (2 * qb + ch) * 1024);
        float dsv[8];
#pragma unroll
        for (int g2 = 0; g2 < 2; ++g2) {
          const f32x4 dl4 = *(const lds_f32x4_t*)(row_at + kDlOff + 4 * (B * BM + qb * 32 + 8 * (2 * ch + g2)));
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            dsv[4 * g2 + jj] = (float)ph[4 * g2 + jj] * (pacc[8 * ch + 4 * g2 + jj] - dl4[jj]);
            dck_part += dsv[4 * g2 + jj];
          }
        }
        const bf16x8 dsb = pack8(dsv);
        lds_wait<0>(tr);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
          acc[db] = mfma32(cat4(tr[2 * db], tr[2 * db + 1]), dsb, acc[db]);
        if constexpr (ch == 0) read_tr(bufc, std::integral_constant<int, 2 * qb + 1>(), tr);
      });
    });
  };

  // step `it`: the P wave on tile `it` (buffer it % 3), the G wave on tile it - 1, tile it + 1
  // loading.  `cur`, `prev`, `ahead`, `ahead2`: the turns of steps it, it - 1, it + 1, it + 2.
  Turn prev{0, 0}, cur{0, 0}, ahead = next(cur), ahead2 = next(ahead);
  auto step = [&](int it, auto bufc) {
    constexpr int B = decltype(bufc)::value;
    constexpr int BN = (B + 1) % 3, BP = (B + 2) % 3;
    if (pwave) wait_all_memory();
    else wait_lds();
    __syncthreads();  // tile `it` and P of tile it - 1 are in LDS
    // a new head: its c at the keys (loaded during the last step of the head before)
    if (pwave && it > 0 && it < total && cur.t == 0)
      ck2 = k_valid ? __builtin_fmaf(next_ckj - next_ck0, kLog2e, -kPkLift) : INFINITY;
    if (it + 1 < total) issue_tile(ahead, std::integral_constant<int, BN>());
    if (it + 2 < total) issue_stats(ahead2, it & 1);
    if (pwave && it + 1 < total && ahead.t == 0) {
      const float* ch = C + row_of(ahead.g);
      next_ck0 = ch[k0];
      next_ckj = k_valid ? ch[kj] : 0.0f;
    }
    if (pwave) {
      if (it < total) {
        const int qt = t_first + cur.t;
        if (qt == t_diag) p_tile(qt, bufc, std::true_type());
        else if (qt > t_diag) p_tile(qt, bufc, std::false_type());
      }
    } else if (it >= 1 && it <= total) {
      if (t_first + prev.t >= t_diag) g_tile(std::integral_constant<int, BP>());
      if (prev.t + 1 == nt) {  // the head ends
        const float tot = wave_sum_pair(dck_part) * kPkUnlift;
        if (k_valid && h == 0) dck[row_of(prev.g) + kj] = -tot;
        dck_part = 0.0f;
      }
    }
    if (it + 1 < total) {
      if (ahead.t == 0) conv_ck0 = next_ck0;
      convert_stats(ahead, (it + 1) & 1, std::integral_constant<int, BN>());
    }
    prev = cur;
    cur = ahead;
    ahead = ahead2;
    ahead2 = next(ahead2);
  };

  issue_stats(cur, 0);
  if (1 < total) issue_stats(ahead, 1);
  issue_tile(cur, std::integral_constant<int, 0>());
  wait_all_memory();
  convert_stats(cur, 0, std::integral_constant<int, 0>());
  for (int it = 0; it <= total; it += 3) {
    step(it, std::integral_constant<int, 0>());
    step(it + 1, std::integral_constant<int, 1>());
    step(it + 2, std::integral_constant<int, 2>());
  }

  const float f = (pwave ? 1.0f : scale) * kPkUnlift;
  if (splits > 1) {
    // partial dK and dV of these heads: [group][dK, dV][Hkv][N][D]
    if (k_valid) {
      float* out = part + (((size_t)hg * 2 + (pwave ? 1 : 0)) * Hkv * N + kv_row + kj) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(out + db * 32 + 8 * g + 4 * h) =
              f32x4{acc[db][4 * g] * f, acc[db][4 * g + 1] * f, acc[db][4 * g + 2] * f,
                    acc[db][4 * g + 3] * f};
    }
  } else if (k_valid) {
    bf16* out = (pwave ? dV : dK) + (kv_row + kj) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 w;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) w[jj] = to_bf16(acc[db][4 * g + jj] * f);
        *reinterpret_cast<bf16x4*>(out + db * 32 + 8 * g + 4 * h) = w;
      }
  }
}

// Groups that the query heads of a key head are split into for dK and dV, a divisor of G.  A
// workgroup walks G / groups heads times the query tiles behind its keys, so the time is about
// the larger of the longest sequence's walk and the mean load of the part, and each split
// writes and reads fp32 sums.  In steps of 128 x 128 scores (bf16: about 3.7 us, one or two
// workgroups per CU at D = 128 and 64; fp32: 32 rows and NW waves, about 8 us per 32 x 32 of
// each wave).
int packed_head_split(bool bf16_, int H, int Hkv, int N, int d, int max_len) {
  const int G = H / Hkv;
  const double rows = bf16_ ? 128 : 32, waves = bf16_ ? 1 : d == 64 ? 8 : 4;
  const double chain = std::max(1.0, max_len / rows / waves), step_us = bf16_ ? 3.7 : 8.0;
  const double mean = (double)H * (N / rows) * (chain + 1) / 2 / (bf16_ && d == 64 ? 512 : 256);
  int best = 1;
  double best_us = 0.0;
  for (int s = 1; s <= G; ++s) {
    if (G % s) continue;
    const double sums = s == 1 ? 0.0 : 5.0 + (double)s * Hkv * N * d * 16 / 4e6;
    const double us = std::max(G / s * chain, mean) * step_us + sums;
    if (s == 1 || us < best_us) {
      best = s;
      best_us = us;
    }
  }
  return best;
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
// Two wave groups (dQ, D = 64: three) share a row block's key tiles where the grid is short and
// the longest row's chain of tiles decides the time: up to two workgroups per CU, counted as
// the rows' blocks, and enough tiles of the longest row to cover the merge.  Forward in
// microseconds, one group / two, H_kv = 4: one sequence of 3001, H = 16, D = 128 62.4 / 50.6 and
// D = 64 41.5 / 33.9; one of 4000, H = 12, D = 64 53.8 / 42.9; four of 1024, H = 8, H_kv = 2, D = 64
// 16.9 / 15.8; beyond two per CU one of 8192, H = 12, D = 64 126.6 / 140.4 and H = 16 151 / 173.
static long long row_blocks(int H, int N) {
  return (long long)H * ((N + kPackedBlock - 1) / kPackedBlock);
}
static bool packed_fwd_split(long long wgs, int max_len) {
  const long long tiles = (max_len + kPkBN - 1) / kPkBN;
  return wgs <= 512 && tiles >= 16 && 16 * tiles >= wgs;
}
// The whole backward with H = H_kv = 4 (so that only dQ is split): 1000 rows, D = 128 73.6 / 69.9,
// D = 64 60.5 / 55.1; 700 rows, D = 128 55.0 / 54.1.
static bool packed_dq_split(long long wgs, int max_len) {
  const long long tiles = (max_len + kPkBN - 1) / kPkBN;
  return wgs <= 512 && tiles >= 8 && 24 * tiles >= wgs;
}

hipError_t launch_packed_fwd(const void* q, const void* k, const void* v, const float* c, void* o,
                             void* o_lo, float* lse, const void* plan, int B, int H, int Hkv,
                             int N, int d, int max_len, float scale, hipStream_t s) {
  const dim3 grid((unsigned)packed_items(B, N) * (unsigned)H);
  auto run = [&](auto kernel, int groups) {
    hipLaunchKernelGGL(kernel, grid, dim3(kPkThreads * groups), 0, s, (const bf16*)q,
                       (const bf16*)k, (const bf16*)v, c, (bf16*)o, (bf16*)o_lo, lse,
                       (const PackedItem*)plan,
                       H, Hkv, N, scale * kLog2e);
  };
  const bool split = packed_fwd_split(row_blocks(H, N), max_len);
  if (d == 128) {
    if (split) run(packed_fwd_kernel<128, 2>, 2);
    else run(packed_fwd_kernel<128, 1>, 1);
  } else {
    if (split) run(packed_fwd_kernel<64, 2>, 2);
    else run(packed_fwd_kernel<64, 1>, 1);
  }
  return hipGetLastError();
}

hipError_t launch_packed_bwd(const void* q, const void* k, const void* v, const float* c,
                             const void* o, const void* o_lo, const float* lse, const void* d_o,
                             void* dq, void* dk, void* dv, float* delta, float* dck, float* part,
                             const void* plan, int B, int H, int Hkv, int N, int d, int max_len,
                             float scale, hipStream_t s) {
  const unsigned items = (unsigned)packed_items(B, N);
  const int splits = packed_head_split(true, H, Hkv, N, d, max_len);
  auto kv = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(items * Hkv * splits), dim3(kPkKvThreads), 0, s, (const bf16*)q,
                       (const bf16*)k, (const bf16*)v, c, lse, (const bf16*)d_o, delta, (bf16*)dk,
                       (bf16*)dv, dck, part, (const PackedItem*)plan, H, Hkv, splits, N, scale,
                       scale * kLog2e);
  };
  const bool split = packed_dq_split(row_blocks(H, N), max_len);
  auto qs = [&](auto kernel, int groups) {
    hipLaunchKernelGGL(kernel, dim3(items * H), dim3(kPkThreads * groups), 0, s, (const bf16*)q,
                       (const bf16*)k, (const bf16*)v, c, lse, (const bf16*)d_o, (const bf16*)o, (const bf16*)o_lo, delta,
                       (bf16*)dq, (const PackedItem*)plan, H, Hkv, N, scale, scale * kLog2e);
  };
  if (d == 128) {
    if (split) qs(packed_dq_kernel<128, kPkDqGroups<128>>, kPkDqGroups<128>);
    else qs(packed_dq_kernel<128, 1>, 1);
    kv(packed_dkdv_kernel<128, 64>);
  } else {
    if (split) qs(packed_dq_kernel<64, kPkDqGroups<64>>, kPkDqGroups<64>);
    else qs(packed_dq_kernel<64, 1>, 1);
    kv(packed_dkdv_kernel<64, 32>);
  }
  return hipGetLastError();
}

}  // namespace fox

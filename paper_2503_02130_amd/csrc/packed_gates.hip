// Packed sequences: the work list of the attention kernels, the gate prefix and its gradient.
//
//   plan      the 128-row blocks of all sequences, most key tiles first (block m of a sequence
//             attends to m + 1 blocks).  Item (s, m) goes to place
//             sum_t max(0, n_t - m - 1) + #{t < s : n_t > m}, n_t the blocks of sequence t:
//             a wave per m finds both by one pass over the lengths, so there is no sort and
//             no atomic.
//   prefix    c = the running sum of log sigmoid(logit) within each sequence, one workgroup
//             per (head, sequence).
//   gradient  d(logit)_l = sigmoid(-logit_l) sum_{i >= l} (dc_q_i + dc_k_i), the same from the
//             sequence's end (without dc_q where it is 0).
//
// The scans run in 64 bits and round once: c of a long sequence is thousands with
// differences of neighbours that matter, and fp32 sums of it are several units off.  They
// are short chains of a few barriers per 8192 rows, bound by latency: sequences of up to 8191
// rows take 7 us, their gradient 12, the plan 4 to 5.  What does not depend on a scan rides on its
// launch: the plan on the prefix's, the sums of split heads (24 us alone beside these 12: 27
// together) and the zeros behind the last sequence on the gradient's.
#include <algorithm>

#include "fox_internal.h"
#include "packed.h"

namespace fox {

constexpr int kPScanThreads = 1024;
constexpr int kPScanPer = 8;
constexpr int kPScanSegment = kPScanThreads * kPScanPer;

// first row and length of sequence b, within [0, N)
__device__ __forceinline__ void packed_range(const int* __restrict__ cu, int b, int N, int& start,
                                             int& len) {
  start = min(max(cu[b], 0), N);
  len = max(min(cu[b + 1], N) - start, 0);
}

// Zeros in the rows behind the last sequence of up to kZeroTensors tensors [heads, N, row], by
// workgroup `group` of kZeroGroups.
struct ZeroList {
  ZeroRows x[kZeroTensors];
  int n;
};
constexpr int kZeroGroups = 64;
static ZeroList zero_list(const ZeroRows* x, int n) {
  ZeroList list;
  list.n = n;
  for (int i = 0; i < n; ++i) list.x[i] = x[i];
  return list;
}
__device__ __forceinline__ void zero_behind(const ZeroList& list, const int* __restrict__ cu, int B,
                                            int N, int group) {
  const int first = min(max(cu[B], 0), N);
  if (first == N) return;
  for (int i = 0; i < list.n; ++i) {
    const ZeroRows z = list.x[i];
    const long long per = (long long)(N - first) * (z.row_bytes / 2);  // 2 bytes divide any row
    for (long long j = (long long)group * blockDim.x + threadIdx.x; j < per * z.heads;
         j += (long long)kZeroGroups * blockDim.x) {
      const long long h = j / per, at = j % per;
      static_cast<uint16_t*>(z.p)[(h * N + first) * (z.row_bytes / 2) + at] = 0;
    }
  }
}
__global__ __launch_bounds__(256) void packed_zero_kernel(ZeroList list, const int* __restrict__ cu,
                                                          int B, int N) {
  zero_behind(list, cu, B, N, (int)blockIdx.x);
}

// dK and dV from the partial sums of groups of heads, in the order of the groups, by workgroup
// `group` of kSumGroups; rows behind the last sequence (no partial sums) are left as they were.
constexpr int kSumGroups = 512;
template <typename T>
__device__ __forceinline__ void head_sum(const HeadSum& x, const int* __restrict__ cu, int B, int N,
                                         int group) {
  const size_t n4 = (size_t)x.Hkv * N * x.d / 4;  // pieces of four of one tensor
  const int end = min(max(cu[B], 0), N);
  for (size_t i = (size_t)group * blockDim.x + threadIdx.x; i < 2 * n4;
       i += (size_t)kSumGroups * blockDim.x) {
    const size_t at = i < n4 ? i : i - n4;
    if ((int)(at / (x.d / 4) % N) >= end) continue;
    f32x4 sum = reinterpret_cast<const f32x4*>(x.part)[i];
    for (int s = 1; s < x.splits; ++s)
      sum += reinterpret_cast<const f32x4*>(x.part)[(size_t)s * 2 * n4 + i];
    T* out = static_cast<T*>(i < n4 ? x.dk : x.dv) + 4 * at;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<bf16x4*>(out) =
          bf16x4{to_bf16(sum[0]), to_bf16(sum[1]), to_bf16(sum[2]), to_bf16(sum[3])};
    } else {
      *reinterpret_cast<f32x4*>(out) = sum;
    }
  }
}

int packed_items(int B, int N) { return N / kPackedBlock + std::min(B, N); }

// The list's places of block number m, by one wave.
struct PlanOut {
  PackedItem* items;
  int n_items, groups;  // workgroups that make it
};
__device__ __forceinline__ void make_plan(const PlanOut& plan, const int* __restrict__ cu, int B, int N,
                                          int m) {
  const int lane = threadIdx.x & 63;
  long long before = 0, total = 0;
  for (int s = lane; s < B; s += 64) {
    int start, len;
    packed_range(cu, s, N, start, len);
    const int nb = (len + kPackedBlock - 1) / kPackedBlock;
    before += max(0, nb - m - 1);
    total += nb;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    before += __shfl_xor(before, off);
    total += __shfl_xor(total, off);
  }
  for (int s0 = 0; s0 < B; s0 += 64) {
    int start = 0, len = 0;
    if (s0 + lane < B) packed_range(cu, s0 + lane, N, start, len);
    const bool has = (len + kPackedBlock - 1) / kPackedBlock > m;
    const uint64_t mask = __ballot(has);
    const long long at = before + __popcll(mask & ((1ull << lane) - 1));
    if (has && at < plan.n_items) plan.items[at] = PackedItem{start, len, m, s0 + lane};
    before += __popcll(mask);
  }
  if (m == 0)
    for (long long i = total + lane; i < plan.n_items; i += 64)
      plan.items[i] = PackedItem{0, 0, 0, -1};
}
// Workgroup `group` of those that make the list, then of those that write zeros.
__device__ __forceinline__ void plan_or_zeros(const PlanOut& plan, const ZeroList& zeros,
                                              const int* __restrict__ cu, int B, int N, int group) {
  if (group < plan.groups)
    make_plan(plan, cu, B, N, group * (int)(blockDim.x >> 6) + (int)(threadIdx.x >> 6));
  else
    zero_behind(zeros, cu, B, N, group - plan.groups);
}
__global__ __launch_bounds__(256) void packed_plan_kernel(const int* __restrict__ cu, int B, int N,
                                                          PlanOut plan, ZeroList zeros) {
  plan_or_zeros(plan, zeros, cu, B, N, (int)blockIdx.x);
}
static PlanOut plan_out(void* plan, int B, int N, int waves) {  // a wave per block number
  const int blocks = (N + kPackedBlock - 1) / kPackedBlock;
  return PlanOut{(PackedItem*)plan, packed_items(B, N), (blocks + waves - 1) / waves};
}

// exp(a), a <= 0, on the transcendental unit: the product with log2(e) in two parts, so that large
// a keep their digits (from -128 on the result is 0, and the parts stay finite).  A NaN stays one
// (a maximum would take the -128), so that a logit that is none shows in c and the gradients.
__device__ __forceinline__ float exp_short(float a) {
  a = a < -128.0f ? -128.0f : a;
  const float y = a * kLog2e;
  const float lo = __builtin_fmaf(a, kLog2e, -y) + a * 1.9259629e-8f;  // log2(e) - float(log2(e))
  const float e = exp2_fast(y);
  return __builtin_fmaf(e, lo * kLn2, e);
}
// log sigmoid(x) = min(x, 0) - log1p(t), t = exp(-|x|), to a few units of the last place:
// log1p(t) = log(u) t / (u - 1) with u = 1 + t rounded (t where u = 1), which cancels the
// rounding of u.  A third of the instructions of expf and log1pf, which bound the scan of a
// long row by one workgroup.
__device__ __forceinline__ float log_sigmoid_short(float x) {
  const float t = exp_short(-fabsf(x));
  const float u = 1.0f + t, d = u - 1.0f;
  const float l = d == 0.0f ? t : __builtin_amdgcn_logf(u) * kLn2 * t * __builtin_amdgcn_rcpf(d);
  return fminf(x, 0.0f) - l;
}
// sigmoid(-x) = 1 / (1 + exp(x)), by the side that does not overflow
__device__ __forceinline__ float sigmoid_neg_short(float x) {
  const float t = exp_short(-fabsf(x));
  return (x > 0.0f ? t : 1.0f) * __builtin_amdgcn_rcpf(1.0f + t);
}

// GRAD false: c from the logits; true: d(logit) from dc_q (may be NULL) and dc_k, and d(log f)
// if aux.  Rows move between memory and LDS one lane beside the other; a thread scans eight
// consecutive ones from there.
template <bool GRAD, typename T>
__global__ __launch_bounds__(kPScanThreads) void packed_scan_kernel(
    const float* __restrict__ dcq, const float* __restrict__ dck, const T* __restrict__ logit,
    const int* __restrict__ cu, float* __restrict__ c, float* __restrict__ aux,
    T* __restrict__ d_logit, int B, int H, int N, ZeroList zeros, HeadSum heads, PlanOut plan) {
  if ((int)blockIdx.x >= B * H) {  // what rides on the launch
    const int other = (int)blockIdx.x - B * H;
    if constexpr (GRAD) {
      const int sums = heads.splits > 1 ? kSumGroups : 0;
      if (other >= sums) zero_behind(zeros, cu, B, N, other - sums);
      else if (heads.bf16) head_sum<bf16>(heads, cu, B, N, other);
      else head_sum<float>(heads, cu, B, N, other);
    } else {
      plan_or_zeros(plan, zeros, cu, B, N, other);
    }
    return;
  }
  __shared__ __attribute__((aligned(16))) float row[kPScanSegment];
  __shared__ double wave_total[kPScanThreads / 64];
  const int b = (int)(blockIdx.x / H), h = (int)(blockIdx.x % H);
  int start, L;
  packed_range(cu, b, N, start, L);
  // the sequence's rows, addressed by 32-bit offsets
  const size_t base = (size_t)h * N + start;
  logit += base;
  if constexpr (GRAD) {
    dck += base;
    d_logit += base;
    if (dcq) dcq += base;
    if (aux) aux += base;
  } else {
    c += base;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  double carry = 0.0;
  for (int seg = 0; seg < L; seg += kPScanSegment) {
    const int m = min(kPScanSegment, L - seg);  // rows of this segment
    // element p of the scan lies at row p, or L - 1 - p from the end
    auto at = [&](int p) { return (unsigned)(GRAD ? L - 1 - p : p); };
#pragma unroll
    for (int e = 0; e < kPScanPer; ++e) {
      const int i = e * kPScanThreads + tid;
      float x = 0.0f;
      if (i < m) {
        const unsigned g = at(seg + i);
        if constexpr (GRAD) x = dcq ? dcq[g] + dck[g] : dck[g];
        else x = log_sigmoid_short((float)logit[g]);
      }
      row[i] = x;
    }
    __syncthreads();
    f32x4* mine = reinterpret_cast<f32x4*>(row) + 2 * tid;
    const f32x4 x0 = mine[0], x1 = mine[1];
    double run[kPScanPer], sum = 0.0;
#pragma unroll
    for (int e = 0; e < kPScanPer; ++e) {
      sum += e < 4 ? x0[e & 3] : x1[e & 3];
      run[e] = sum;
    }
    double incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const double y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    if (lane == 63) wave_total[wave] = incl;
    // The sum of the lanes before this one, not incl - sum: a term of the lane's own that is
    // far larger (a gate that forgets everything) or not finite would take them with it.
    const double lanes = __shfl_up(incl, 1);
    __syncthreads();
    double prior = carry + (lane ? lanes : 0.0);
#pragma unroll
    for (int w = 0; w < kPScanThreads / 64; ++w) {
      if (w < wave) prior += wave_total[w];
      carry += wave_total[w];
    }
    f32x4 y0, y1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y0[e] = (float)(prior + run[e]);
      y1[e] = (float)(prior + run[4 + e]);
    }
    mine[0] = y0;
    mine[1] = y1;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPScanPer; ++e) {
      const int i = e * kPScanThreads + tid;
      if (i < m) {
        const unsigned g = at(seg + i);
        const float y = row[i];
        if constexpr (GRAD) {
          if (aux) aux[g] = y;
          d_logit[g] = (T)(y * sigmoid_neg_short((float)logit[g]));
        } else {
          c[g] = y;
        }
      }
    }
    __syncthreads();  // the next segment writes the rows again
  }
}

hipError_t launch_packed_plan(const int* cu, int B, int N, void* plan, const ZeroRows* zeros,
                              int n_zeros, hipStream_t s) {
  const PlanOut out = plan_out(plan, B, N, 4);
  hipLaunchKernelGGL(packed_plan_kernel, dim3(out.groups + (n_zeros ? kZeroGroups : 0)), dim3(256), 0,
                     s, cu, B, N, out, zero_list(zeros, n_zeros));
  return hipGetLastError();
}

hipError_t launch_packed_prefix(bool bf16_, const void* logit, const int* cu, float* c, int B,
                                int H, int N, void* plan, const ZeroRows* zeros, int n_zeros,
                                hipStream_t s) {
  const PlanOut out = plan ? plan_out(plan, B, N, kPScanThreads / 64) : PlanOut{};
  const dim3 grid((unsigned)B * (unsigned)H + out.groups + (n_zeros ? kZeroGroups : 0)),
      block(kPScanThreads);
  if (bf16_)
    hipLaunchKernelGGL((packed_scan_kernel<false, bf16>), grid, block, 0, s, nullptr, nullptr,
                       (const bf16*)logit, cu, c, nullptr, nullptr, B, H, N,
                       zero_list(zeros, n_zeros), HeadSum{}, out);
  else
    hipLaunchKernelGGL((packed_scan_kernel<false, float>), grid, block, 0, s, nullptr, nullptr,
                       (const float*)logit, cu, c, nullptr, nullptr, B, H, N,
                       zero_list(zeros, n_zeros), HeadSum{}, out);
  return hipGetLastError();
}

hipError_t launch_packed_gate_grad(bool bf16_, const float* dcq, const float* dck,
                                   const void* logit, const int* cu, float* d_log_f,
                                   void* d_logit, int B, int H, int N, const HeadSum& sum,
                                   const ZeroRows* zeros, int n_zeros, hipStream_t s) {
  const dim3 grid((unsigned)B * (unsigned)H + (sum.splits > 1 ? kSumGroups : 0) +
                  (n_zeros ? kZeroGroups : 0)),
      block(kPScanThreads);
  if (bf16_)
    hipLaunchKernelGGL((packed_scan_kernel<true, bf16>), grid, block, 0, s, dcq, dck,
                       (const bf16*)logit, cu, nullptr, d_log_f, (bf16*)d_logit, B, H, N,
                       zero_list(zeros, n_zeros), sum, PlanOut{});
  else
    hipLaunchKernelGGL((packed_scan_kernel<true, float>), grid, block, 0, s, dcq, dck,
                       (const float*)logit, cu, nullptr, d_log_f, (float*)d_logit, B, H, N,
                       zero_list(zeros, n_zeros), sum, PlanOut{});
  return hipGetLastError();
}

hipError_t launch_packed_zero(const ZeroRows* x, int n, const int* cu, int B, int N,
                              hipStream_t s) {
  hipLaunchKernelGGL(packed_zero_kernel, dim3(kZeroGroups), dim3(256), 0, s, zero_list(x, n), cu, B,
                     N);
  return hipGetLastError();
}

}  // namespace fox

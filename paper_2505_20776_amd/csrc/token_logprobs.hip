// What a verification step reads from a row of logits: the most probable tokens (the first of them is the token that greedy
// acceptance wants), the log-sum-exp, the entropy, and the log probabilities of given tokens.
//
//   x = logit_scale l;  lse = m + ln Z,  Z = sum e^(x - m);  entropy = ln Z - (sum e^(x - m) (x - m)) / Z;  log p(t) = (x_t - m) - ln Z
//
// The logits are read once: a workgroup holds a slice of a row (512 threads x up to 64 values) in registers, so that the maximum
// is known before the exponentials, and m is the slice's.  Long rows are several slices, joined by a second launch.
//
// The k largest of a slice: a value and its index make one 64-bit key (larger values first, the lower index among equal ones),
// so all keys differ and every answer is unique.  Each group of eight lanes finds its largest key; the k-th largest of these 64
// keys has at least k keys at or above it, and few more: 20 of 32768 random values for k = 16.  Those are listed in LDS, and a
// key whose rank in the list is r goes to place r.  A list that would overflow (values that crowd in few groups) has its
// threshold raised by bisection first.
#include "mfma_util.h"
#include "token_logprobs.h"

namespace specext {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kList = 1024;             // keys that the list of a slice holds
constexpr int kJoinThreads = 256;

using Key = unsigned long long;

// order-preserving bits of a float; 0 is below all of them.  NaN is the largest, -0 equals 0.
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order_bits(uint32_t b) {
  return __uint_as_float(b == 0xffffffffu ? 0x7fc00000u : b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ Key make_key(float x, int index) {
  return (static_cast<Key>(order_bits(x)) << 32) | (0xffffffffu - static_cast<uint32_t>(index));
}
__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key key_from_lane(Key k, int mask) {
  const uint32_t lo = __shfl_xor(static_cast<uint32_t>(k), mask, 64), hi = __shfl_xor(static_cast<uint32_t>(k >> 32), mask, 64);
  return (static_cast<Key>(hi) << 32) | lo;
}

struct RowStats {
  float m, z, w;      // maximum, sum of e^(x - m), sum of e^(x - m) (x - m)
};

// the last step: what the caller asked for of one row, from its sums and its k best keys in LDS
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int row, RowStats s, const Key* best, int n_best, int tid, int threads) {
  const bool empty = s.m == -INFINITY && s.z == 0.f;       // nothing but minus infinity
  const float ln_z = logf(s.z);
  const float lse = empty ? -INFINITY : s.m + ln_z;
  if (tid == 0) {
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = empty ? 0.f : ln_z - s.w / s.z;
  }
  for (int i = tid; i < n_best; i += threads) {
    const float x = from_order_bits(static_cast<uint32_t>(best[i] >> 32));
    a.top_id[static_cast<int64_t>(row) * a.k + i] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(best[i]));
    if (a.top_logprob) a.top_logprob[static_cast<int64_t>(row) * a.k + i] = empty ? -INFINITY : (x - s.m) - ln_z;
  }
  for (int i = tid; i < a.n_given; i += threads) {
    const int token = a.tokens[static_cast<int64_t>(row) * a.n_given + i];
    float lp = -INFINITY;                         // no token of the vocabulary
    if (token >= 0 && token < a.vocab && !empty) {
      const int64_t at = row * a.row_stride + token;
      lp = ((a.bf16 ? bf16_bits_to_float(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at]) * a.logit_scale - s.m) - ln_z;
    }
    a.logprob[static_cast<int64_t>(row) * a.n_given + i] = lp;
  }
}

// ranks of `n` keys in LDS, all different; the k largest to out in order
__device__ __forceinline__ void rank_keys(const Key* list, int n, int k, Key* out, int tid, int threads) {
  for (int i = tid; i < n; i += threads) {
    const Key mine = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > mine ? 1 : 0;
    if (rank < k) out[rank] = mine;
  }
}

// One slice of one row.  E values per thread; slice `s` holds the 16-byte vectors [s, s + 1) x kThreads x (E / V) of the row, counted
// from the row's first address rounded down to 16 bytes.
template <bool BF16, int E, bool ONE>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobArgs a) {
  constexpr int V = BF16 ? 8 : 4;                 // values per vector
  constexpr int N = E / V;
  __shared__ float part[3][kWaves];
  __shared__ Key group_best[64];
  __shared__ Key list[kList];
  __shared__ Key best[64];
  __shared__ int counts[kWaves];
  __shared__ int listed;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = ONE ? blockIdx.x : blockIdx.x / a.slices;
  const int slice = ONE ? 0 : blockIdx.x - row * a.slices;
  const unsigned char* base = static_cast<const unsigned char*>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(base) & 15) / (BF16 ? 2 : 4);   // values in front of the row in its first vector
  base -= lead * (BF16 ? 2 : 4);

  // first[i]: index of vector i's first value; values outside [0, vocab) are absent
  float x[E];
  auto first_of = [&](int i) { return (slice * N * kThreads + i * kThreads + tid) * V - lead; };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int first = first_of(i);
    const unsigned char* at = base + static_cast<int64_t>(first + lead) * (BF16 ? 2 : 4);
    if (first >= 0 && first + V <= a.vocab) {
      const uintx4 w = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(at));
#pragma unroll
      for (int e = 0; e < V; ++e)
        x[i * V + e] = BF16 ? __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16) : __uint_as_float(w[e & 3]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[i * V + e] = -INFINITY;
        if (first + e >= 0 && first + e < a.vocab)
          x[i * V + e] = BF16 ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(at)[e]) : reinterpret_cast<const float*>(at)[e];
      }
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] *= a.logit_scale;
    top = fmaxf(top, x[e]);
  }
  top = wave_max(top);
  if (lane == 0) part[0][wave] = top;
  if (tid == 0) listed = 0;
  if (tid < 64) best[tid] = 0;

  // this thread's largest key, then its group's
  const int k = a.k;
  Key mine = 0;
  if (k > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int index = first_of(i) + e;
        const Key key = make_key(x[i * V + e], index);
        if (index >= 0 && index < a.vocab) mine = max_key(mine, key);
      }
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) mine = max_key(mine, key_from_lane(mine, m));
    if ((lane & 7) == 0) group_best[tid >> 3] = mine;
  }
  __syncthreads();
  RowStats st;
  st.m = part[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) st.m = fmaxf(st.m, part[0][w]);
  const float m = st.m == -INFINITY ? 0.f : st.m;
  float z = 0.f, wsum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float d = x[e] - m;
    const float t = fast_exp2(d * kLog2e);
    z += t;
    wsum = fmaf(t, d < -1e4f ? -1e4f : d, wsum);    // 0 x -inf is 0 here; a NaN stays
  }
  z = wave_sum(z);
  wsum = wave_sum(wsum);
  if (lane == 0) {
    part[1][wave] = z;
    part[2][wave] = wsum;
  }

  if (k > 0) {
    // threshold: the k-th largest of the 64 group keys (0, every key, where fewer groups have any)
    const Key own = group_best[lane];
    int rank = 0;
    for (int j = 0; j < 64; ++j) rank += group_best[j] > own ? 1 : 0;
    const unsigned long long at_k = __ballot(rank == k - 1 && own != 0);
    Key threshold = 0;
    if (at_k) {
      const int from = __builtin_ctzll(at_k);
      threshold = group_best[from];
    }
    auto count_from = [&](Key from) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int index = first_of(i) + e;
          n += index >= 0 && index < a.vocab && make_key(x[i * V + e], index) >= from ? 1 : 0;
        }
      n = static_cast<int>(wave_sum(static_cast<float>(n)));      // at most 4096: exact
      __syncthreads();
      if (lane == 0) counts[wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) n += counts[w];
      return n;
    };
    if (__builtin_expect(count_from(threshold) > kList, 0)) {
      // the largest threshold with at least k keys has exactly k
      Key lo = threshold, hi = ~Key{0};           // at least k keys from lo on, fewer than k from hi on
      while (hi - lo > 1) {
        const Key mid = lo + (hi - lo) / 2;
        if (count_from(mid) >= k) lo = mid;
        else hi = mid;
      }
      threshold = lo;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int index = first_of(i) + e;
        const Key key = make_key(x[i * V + e], index);
        if (index >= 0 && index < a.vocab && key >= threshold) list[atomicAdd(&listed, 1)] = key;
      }
  }
  __syncthreads();
  st.z = 0.f, st.w = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    st.z += part[1][w];
    st.w += part[2][w];
  }
  if (k > 0) rank_keys(list, listed, k, best, tid, kThreads);
  __syncthreads();
  if constexpr (ONE) {
    finish_row(a, row, st, best, k, tid, kThreads);
  } else {
    const int64_t at = static_cast<int64_t>(row) * a.slices + slice;
    if (tid == 0) *reinterpret_cast<floatx4*>(a.stats + at * 4) = floatx4{st.m, st.z, st.w, 0.f};
    if (tid < k) a.keys[at * k + tid] = best[tid];
  }
}

// the slices of one row
__global__ __launch_bounds__(kJoinThreads) void logprobs_join_kernel(LogprobArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  Key* list = reinterpret_cast<Key*>(lds);        // slices x k, then k best
  const int tid = threadIdx.x;
  const int row = blockIdx.x;
  const int n = a.slices * a.k;
  Key* best = list + n;
  for (int i = tid; i < n; i += kJoinThreads) list[i] = a.keys[static_cast<int64_t>(row) * n + i];
  RowStats s = {-INFINITY, 0.f, 0.f};
  for (int i = 0; i < a.slices; ++i) s.m = fmaxf(s.m, a.stats[(static_cast<int64_t>(row) * a.slices + i) * 4]);
  for (int i = 0; i < a.slices; ++i) {
    const floatx4 t = *reinterpret_cast<const floatx4*>(a.stats + (static_cast<int64_t>(row) * a.slices + i) * 4);
    if (t[0] == -INFINITY && t[1] == 0.f) continue;         // nothing but minus infinity
    const float d = t[0] - s.m;
    const float f = fast_exp2(d * kLog2e);
    s.z = fmaf(t[1], f, s.z);
    s.w = fmaf(f, fmaf(d < -1e4f ? -1e4f : d, t[1], t[2]), s.w);
  }
  __syncthreads();
  // short slices leave zeros behind their keys; every row has k keys at least, and zeros rank behind all of them
  rank_keys(list, n, a.k, best, tid, kJoinThreads);
  __syncthreads();
  finish_row(a, row, s, best, a.k, tid, kJoinThreads);
}

template <bool BF16, bool ONE>
hipError_t launch_slices(const LogprobArgs& a, int per_thread, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.n_rows) * a.slices), block(kThreads);
  switch (per_thread) {
    case 8: return launch_kernel(logprobs_kernel<BF16, 8, ONE>, grid, block, 0, stream, a);
    case 16: return launch_kernel(logprobs_kernel<BF16, 16, ONE>, grid, block, 0, stream, a);
    case 32: return launch_kernel(logprobs_kernel<BF16, 32, ONE>, grid, block, 0, stream, a);
    default: return launch_kernel(logprobs_kernel<BF16, 64, ONE>, grid, block, 0, stream, a);
  }
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobArgs& a, int per_thread, hipStream_t stream) {
  if (a.n_rows <= 0) return hipSuccess;
  hipError_t e;
  if (a.slices == 1) return a.bf16 ? launch_slices<true, true>(a, per_thread, stream) : launch_slices<false, true>(a, per_thread, stream);
  e = a.bf16 ? launch_slices<true, false>(a, per_thread, stream) : launch_slices<false, false>(a, per_thread, stream);
  if (e != hipSuccess) return e;
  const int lds_bytes = (a.slices + 1) * a.k * static_cast<int>(sizeof(Key));
  return launch_kernel(logprobs_join_kernel, dim3(a.n_rows), dim3(kJoinThreads), lds_bytes, stream, a);
}

}  // namespace specext

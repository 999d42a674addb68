// What a verification step reads from a row of logits: the most probable tokens (the first of them is the token that greedy
// acceptance wants), the log-sum-exp, the entropy, and the log probabilities of given tokens.
//
//   m = max l,  t = e^(s (l - m)),  Z = sum t,  lse = s m + ln Z,  entropy = ln Z - s (sum t (l - m)) / Z,
//   log p(i) = s (l_i - m) - ln Z                         (s = logit_scale)
//
// The logits are read once: a workgroup holds a slice of a row (512 threads x up to eight 16-byte vectors) in registers, bf16 as it
// came, so that the maximum is known before the exponentials.  Long rows are several slices, joined by a second launch.
//
// Many rows are bound by memory and, next to it, by the two passes of the vector ALUs over every value (maximum; exponential and
// sums): 2048 bf16 rows of 128256, eight answers, 525 MB, 107 us and 4.8 for the join, 4.9 TB/s (a plain read 7.1).  Few rows are
// bound by latency, two launches of one load and some twenty exchanges between lanes: one fp32 row of 32000 4.3 + 3.1 us, 60 bf16
// rows of 128256 7.8 + 3.1.
//
// The k largest of a slice: a value and its index make one 64-bit key (larger values first, the lower index among equal ones), so all
// keys differ and every answer is unique.  Each wave, or for more than eight answers each group of eight lanes, has its largest value,
// which the softmax needs anyway; at or above the k-th largest of these are at least k values, and few more: about 20 of 32768 random
// ones for k = 8, and for k = 16.  Those are listed in LDS, found through the maxima of the vectors, and a key whose rank in the
// list is r goes to place r.  Values that crowd (many equal ones, a run of large ones in one group) overflow the list; the threshold
// is then the k-th largest of the 512 threads' own best keys, and if that is not enough found by bisection.
#include "mfma_util.h"
#include "token_logprobs.h"

namespace specext {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kList = 1024;             // keys that the list of a slice holds
constexpr int kJoinThreads = 256;
constexpr float kLargest = 3.402823466e38f;

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
  float m, z, w;      // maximum, sum of t, sum of t (l - m)
};

// the last step: what the caller asked for of one row, from its sums and its k best keys in LDS
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int row, RowStats s, const Key* best, int n_best, int tid, int threads) {
  const bool empty = s.m == -INFINITY && s.z == 0.f;       // nothing but minus infinity
  const float ln_z = logf(s.z);
  if (tid == 0) {
    if (a.lse) a.lse[row] = empty ? -INFINITY : fmaf(a.logit_scale, s.m, ln_z);
    if (a.entropy) a.entropy[row] = empty ? 0.f : ln_z - a.logit_scale * (s.w / s.z);
  }
  for (int i = tid; i < n_best; i += threads) {
    const float x = from_order_bits(static_cast<uint32_t>(best[i] >> 32));
    a.top_id[static_cast<int64_t>(row) * a.k + i] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(best[i]));
    if (a.top_logprob) a.top_logprob[static_cast<int64_t>(row) * a.k + i] = empty ? -INFINITY : fmaf(a.logit_scale, x - s.m, -ln_z);
  }
  for (int i = tid; i < a.n_given; i += threads) {
    const int token = a.tokens[static_cast<int64_t>(row) * a.n_given + i];
    float lp = -INFINITY;                         // no token of the vocabulary
    if (token >= 0 && token < a.vocab && !empty) {
      const int64_t at = row * a.row_stride + token;
      const float x = a.bf16 ? bf16_bits_to_float(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
      lp = fmaf(a.logit_scale, x - s.m, -ln_z);
    }
    a.logprob[static_cast<int64_t>(row) * a.n_given + i] = lp;
  }
}

// The k largest of n keys in LDS, all different, to out in order.  The list has room for kRankStep keys more, which are cleared here:
// the comparisons read whole steps, all their reads under way at once.
constexpr int kRankStep = 16;
template <bool ONE_WAVE = false>
__device__ __forceinline__ void rank_keys(Key* list, int n, int k, Key* out, int tid, int threads) {
  typedef __attribute__((ext_vector_type(2))) Key Key2;
  if (tid < kRankStep) list[n + tid] = 0;
  if (ONE_WAVE) __builtin_amdgcn_wave_barrier();
  else __syncthreads();
  for (int i = tid; i < n; i += threads) {
    const Key mine = list[i];
    int rank = 0;
    for (int j = 0; j < n; j += kRankStep) {
      Key2 other[kRankStep / 2];
#pragma unroll
      for (int u = 0; u < kRankStep / 2; ++u) other[u] = reinterpret_cast<const Key2*>(list + j)[u];
#pragma unroll
      for (int u = 0; u < kRankStep / 2; ++u) rank += (other[u][0] > mine ? 1 : 0) + (other[u][1] > mine ? 1 : 0);
    }
    if (rank < k) out[rank] = mine;
  }
}

// One slice of one row: N 16-byte vectors per thread.  Slice i holds the vectors [i, i + 1) x kThreads x N of the row, counted from the
// row's first address rounded down to 16 bytes.
template <bool BF16, int N, bool ONE>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobArgs a) {
  constexpr int V = BF16 ? 8 : 4;                 // values per vector
  constexpr int kBytes = BF16 ? 2 : 4;
  __shared__ float part[2][kWaves];
  __shared__ float group_top[64], wave_top[kWaves];
  __shared__ float threshold_of;
  __shared__ __attribute__((aligned(16))) Key list[kList + kRankStep];
  __shared__ Key best[64];
  __shared__ int counts[kWaves];
  __shared__ int listed;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = ONE ? blockIdx.x : blockIdx.x / a.slices;
  const int slice = ONE ? 0 : blockIdx.x - row * a.slices;
  const unsigned char* base = static_cast<const unsigned char*>(a.logits) + row * a.row_stride * kBytes;
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(base) & 15) / kBytes;   // values in front of the row in its first vector
  base -= lead * kBytes;

  // values of a vector that lie outside the row are minus infinity here, and are told apart by their index where that matters
  uintx4 w[N];
  auto first_of = [&](int i) { return (slice * N * kThreads + i * kThreads + tid) * V - lead; };
  auto value = [&](const uintx4& v, int e) {
    return BF16 ? __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16) : __uint_as_float(v[e & 3]);
  };
  // widened values and keys are made anew in every pass, instead of kept in as many registers again
  auto forget = [&](uintx4& v) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t u = v[c];
      asm volatile("" : "+v"(u));
      v[c] = u;
    }
  };
  auto in_row = [&](int index) { return index >= 0 && index < a.vocab; };
  auto load_vector = [&](int i) {
    const int first = first_of(i);
    const unsigned char* at = base + static_cast<int64_t>(first + lead) * kBytes;
    if (first >= 0 && first + V <= a.vocab) return __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(at));
    uint32_t u[4] = {};
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (BF16) {
        const uint32_t x = in_row(first + e) ? reinterpret_cast<const uint16_t*>(at)[e] : 0xff80u;
        u[e >> 1] |= x << (16 * (e & 1));
      } else {
        u[e] = in_row(first + e) ? reinterpret_cast<const uint32_t*>(at)[e] : 0xff800000u;
      }
    }
    return uintx4{u[0], u[1], u[2], u[3]};
  };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // all 512 vectors inside the row: no lane looks at its own place
    const int first = (slice * N + i) * kThreads * V - lead;
    if (__builtin_expect(first >= 0 && first + kThreads * V <= a.vocab, 1))
      w[i] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(base + static_cast<int64_t>(first_of(i) + lead) * kBytes));
    else
      w[i] = load_vector(i);
  }
  const int k = a.k;
  if (tid == 0) listed = 0;
  if (tid < 64) best[tid] = 0;
  float top[N];                                   // of each vector
  float mine = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    top[i] = value(w[i], 0);
#pragma unroll
    for (int e = 1; e < V; ++e) top[i] = fmaxf(top[i], value(w[i], e));
    mine = fmaxf(mine, top[i]);
  }
  // the largest values of eight lanes and of the wave
  mine = fmaxf(mine, SPECEXT_DPP(mine, 0xB1));
  mine = fmaxf(mine, SPECEXT_DPP(mine, 0x4E));
  mine = fmaxf(mine, SPECEXT_DPP(mine, 0x141));
  if ((lane & 7) == 0) group_top[tid >> 3] = mine;
  mine = wave_max(mine);
  if (lane == 0) wave_top[wave] = mine;
  __syncthreads();
  const float of_wave = wave_top[lane & (kWaves - 1)];
  RowStats st = {wave_max(of_wave), 0.f, 0.f};
  // The threshold: the largest value that k groups reach.  For up to eight answers a group is a wave, unless too few waves have
  // values (a short slice); else eight lanes, found by one wave while the others take exponentials.
  auto of_groups = [&]() __attribute__((always_inline)) {
    const float group = group_top[lane];
    int reach = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) reach += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(group), j)) >= group ? 1 : 0;
    return wave_max(reach >= k ? group : -INFINITY);
  };
  const bool few = k <= kWaves;
  float threshold = st.m;
  if (few) {
    int reach = 0;
#pragma unroll
    for (int j = 0; j < kWaves; ++j) reach += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(of_wave), j)) >= of_wave ? 1 : 0;
    threshold = wave_max(reach >= k ? of_wave : -INFINITY);
    if (__builtin_expect(threshold == -INFINITY && k > 0, 0)) threshold = of_groups();
  } else if (wave == 0) {
    const float reached = of_groups();
    if (lane == 0) threshold_of = reached;
  }
  const float m = st.m == -INFINITY ? 0.f : st.m;
  const float to_log2 = a.logit_scale * kLog2e;
  float z = 0.f, wsum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    forget(w[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = value(w[i], e) - m;
      const float t = fast_exp2(d * to_log2);
      z += t;
      wsum = fmaf(t, fmaxf(d, -kLargest), wsum);          // nothing times minus infinity is nothing here; t of a NaN is one
    }
  }
  z = wave_sum(z);
  wsum = wave_sum(wsum);
  if (lane == 0) {
    part[0][wave] = z;
    part[1][wave] = wsum;
  }
  if (!few) {
    __syncthreads();
    threshold = threshold_of;
  }
  if (k > 0) {
    // Fewer than k groups with anything but minus infinity: everything else there is, and the first k values of the slice, among
    // which are as many of the minus infinities as are wanted, of the lowest indices.
    const int slice_first = slice * N * kThreads * V - lead;
    const int equal_end = threshold == -INFINITY ? (slice_first < 0 ? 0 : slice_first) + k : 0x7fffffff;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (top[i] >= threshold) {
        forget(w[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float x = value(w[i], e);
          if (x >= threshold) {
            const int index = first_of(i) + e;
            if ((x > threshold || index < equal_end) && in_row(index)) {
              const int place = atomicAdd(&listed, 1);
              if (place < kList) list[place] = make_key(x, index);
            }
          }
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    st.z += part[0][v];
    st.w += part[1][v];
  }
  const int64_t at = ONE ? row : static_cast<int64_t>(row) * a.slices + slice;
  if (__builtin_expect(listed <= 128 && st.z == st.z, 1)) {
    // a short list, as a rule: one wave ranks it, the others leave their place to the next workgroup
    if (wave != 0) return;
    if (k > 0) rank_keys<true>(list, listed, k, best, lane, 64);
    __builtin_amdgcn_wave_barrier();
    if constexpr (ONE) {
      finish_row(a, row, st, best, k, lane, 64);
    } else {
      if (lane == 0) *reinterpret_cast<floatx4*>(a.stats + at * 4) = floatx4{st.m, st.z, st.w, 0.f};
      if (lane < k) a.keys[at * k + lane] = best[lane];
    }
    return;
  }
  if (k > 0) {
    if (__builtin_expect(listed > kList || st.z != st.z, 0)) {
      // too many, or a NaN, which no maximum shows: by keys, from the slice as it is in memory
      auto count_from = [&](Key from) {
        int n = 0;
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
          const uintx4 v = load_vector(i);
#pragma unroll
          for (int e = 0; e < V; ++e) n += in_row(first_of(i) + e) && make_key(value(v, e), first_of(i) + e) >= from ? 1 : 0;
        }
        n = static_cast<int>(wave_sum(static_cast<float>(n)));      // at most 4096: exact
        __syncthreads();
        if (lane == 0) counts[wave] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) n += counts[v];
        return n;
      };
      Key own = 0;
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const uintx4 v = load_vector(i);
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (in_row(first_of(i) + e)) own = max_key(own, make_key(value(v, e), first_of(i) + e));
      }
      __syncthreads();
      list[tid] = own;
      __syncthreads();
      // (best holds zeros: the threshold is 0, every key, where fewer than k threads have any)
      rank_keys(list, kThreads, k, best, tid, kThreads);
      __syncthreads();
      Key lo = best[k - 1], hi = ~Key{0};
      if (count_from(lo) > kList) {
        // the largest threshold with at least k keys has exactly k
        while (hi - lo > 1) {
          const Key mid = lo + (hi - lo) / 2;
          if (count_from(mid) >= k) lo = mid;
          else hi = mid;
        }
      }
      __syncthreads();
      if (tid == 0) listed = 0;
      if (tid < 64) best[tid] = 0;
      __syncthreads();
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const uintx4 v = load_vector(i);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int index = first_of(i) + e;
          const Key key = make_key(value(v, e), index);
          if (in_row(index) && key >= lo) list[atomicAdd(&listed, 1)] = key;
        }
      }
      __syncthreads();
    }
    rank_keys(list, listed, k, best, tid, kThreads);
    __syncthreads();
  }
  if constexpr (ONE) {
    finish_row(a, row, st, best, k, tid, kThreads);
  } else {
    if (tid == 0) *reinterpret_cast<floatx4*>(a.stats + at * 4) = floatx4{st.m, st.z, st.w, 0.f};
    if (tid < k) a.keys[at * k + tid] = best[tid];
  }
}

// The slices of one row: a lane has one of them.
__global__ __launch_bounds__(kJoinThreads) void logprobs_join_kernel(LogprobArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int row = blockIdx.x;
  const int n = a.slices * a.k;
  Key* list = reinterpret_cast<Key*>(lds);        // n keys, kRankStep more, then the k best
  Key* best = list + n + kRankStep;
  static_assert(kMaxSlices <= 64, "a slice per lane");
  floatx4 t = {-INFINITY, 0.f, 0.f, 0.f};
  if (lane < a.slices) t = *reinterpret_cast<const floatx4*>(a.stats + (static_cast<int64_t>(row) * a.slices + lane) * 4);
  for (int i = tid; i < n; i += kJoinThreads) list[i] = a.keys[static_cast<int64_t>(row) * n + i];
  RowStats s;
  s.m = wave_max(t[0]);
  // a slice of nothing but minus infinity adds nothing (nor does it where the whole row is that)
  const float d = t[0] == s.m ? 0.f : t[0] - s.m;
  const float f = fast_exp2(d * a.logit_scale * kLog2e);
  s.z = wave_sum(t[1] * f);
  s.w = wave_sum(f > 0.f ? f * fmaf(d, t[1], t[2]) : 0.f);
  // short slices leave zeros behind their keys; every row has k keys at least, and zeros rank behind all of them
  if (a.k > 0) rank_keys(list, n, a.k, best, tid, kJoinThreads);
  __syncthreads();
  finish_row(a, row, s, best, a.k, tid, kJoinThreads);
}

template <bool BF16, bool ONE>
hipError_t launch_slices(const LogprobArgs& a, int vectors, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.n_rows) * a.slices), block(kThreads);
  switch (vectors) {
    case 1: return launch_kernel(logprobs_kernel<BF16, 1, ONE>, grid, block, 0, stream, a);
    case 2: return launch_kernel(logprobs_kernel<BF16, 2, ONE>, grid, block, 0, stream, a);
    case 4: return launch_kernel(logprobs_kernel<BF16, 4, ONE>, grid, block, 0, stream, a);
    default: return launch_kernel(logprobs_kernel<BF16, 8, ONE>, grid, block, 0, stream, a);
  }
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobArgs& a, int vectors, hipStream_t stream) {
  if (a.n_rows <= 0) return hipSuccess;
  if (a.slices == 1) return a.bf16 ? launch_slices<true, true>(a, vectors, stream) : launch_slices<false, true>(a, vectors, stream);
  const hipError_t e = a.bf16 ? launch_slices<true, false>(a, vectors, stream) : launch_slices<false, false>(a, vectors, stream);
  if (e != hipSuccess) return e;
  const int lds_bytes = ((a.slices + 1) * a.k + kRankStep) * static_cast<int>(sizeof(Key));
  return launch_kernel(logprobs_join_kernel, dim3(a.n_rows), dim3(kJoinThreads), lds_bytes, stream, a);
}

}  // namespace specext

// The target cache in 8 bits: rows go in (a prompt's, or the accepted rows of a draft tree), and come back out.
//
//   scale[b] = 2^e, the smallest with  max |x| <= 448 2^e  over the new rows of block b  (e >= -100), or the scale that the
//              block has, where it holds older rows and that one is larger
//   code     = e4m3(x / scale), to the nearest, ties to even;  x = code scale
//
// A power of two only moves the exponent of a code, so rows that are there already lose nothing when a later one needs a larger
// scale (codes that leave the normal range, 2^-6 and more, round to steps of 2^-9).
//
// One workgroup has one block of one head, of K or of V: it holds the block's new rows in registers, finds their largest
// magnitude, and writes codes and scale, so the rows are read once and no two workgroups share a scale.
//
// Bound by memory for prompts: 8192 bf16 tokens of 32 layers with 8 128-wide heads, 1.6 GB read and written, 297 us to write and 299
// to read back, 5.4 TB/s (a copy of 2 GiB: 4.85).  By latency for the accepted rows of a tree, five of them over those 32 layers
// 4.8 us, most of it a launch and three loads that wait for one another: count, path, rows.
#include "mfma_util.h"
#include "quant_cache.h"

namespace specext {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// 16 values of a row as fp32
template <bool BF16>
struct Piece {
  uintx4 w[BF16 ? 2 : 4];
  __device__ __forceinline__ void load(const void* src) {
#pragma unroll
    for (int i = 0; i < (BF16 ? 2 : 4); ++i) w[i] = static_cast<const uintx4*>(src)[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (BF16 ? 2 : 4); ++i) w[i] = uintx4{0, 0, 0, 0};
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (BF16) {
      const uint32_t v = w[e >> 3][(e >> 1) & 3];
      return __uint_as_float(e & 1 ? v & 0xffff0000u : v << 16);
    } else {
      return __uint_as_float(w[e >> 2][e & 3]);
    }
  }
};

__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true));
}

__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = part[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part[w]);
  return m;
}

// D: head_dim; ITEMS: 16-value pieces of a block per thread
template <int D, bool BF16, int ITEMS>
__global__ __launch_bounds__(kThreads) void quant_write_kernel(QuantWrite a) {
  __shared__ float part[2][kWaves];
  constexpr int kPieces = D / 16;                 // of a row
  const int lh = blockIdx.y;
  const int layer = lh / a.n_kv_heads, g = lh - layer * a.n_kv_heads;
  const bool is_v = blockIdx.z != 0;
  const int first_block = a.start >> a.block_log2;
  const int block = first_block + blockIdx.x;
  const int pos0 = block << a.block_log2;         // position of the block's first row
  int n = a.n_tokens;
  if (a.n_accept) {
    n = *a.n_accept;
    n = n < 0 ? 0 : n < a.n_tokens ? n : a.n_tokens;
  }
  const int end = a.start + n;
  if (n == 0 || pos0 >= end) return;
  const unsigned char* src = static_cast<const unsigned char*>(is_v ? a.v_src : a.k_src) + layer * a.src_sy + g * a.src_sh;
  unsigned char* cache = static_cast<unsigned char*>(is_v ? a.v_cache : a.k_cache) + layer * a.cache_sy + g * a.cache_sh;
  float* scale_at = (is_v ? a.v_scale : a.k_scale) + layer * a.scale_sy + g * a.scale_sh + block;
  const int rows = 1 << a.block_log2;
  const bool has_older = pos0 < a.start;
  const float old_scale = has_older ? *scale_at : 0.f;

  Piece<BF16> x[ITEMS];
  bool fresh[ITEMS];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int item = i * kThreads + threadIdx.x;
    const int row = item / kPieces;
    const int pos = pos0 + row;
    const int from = quant_source_row(row < rows && pos >= a.start && pos < end ? pos - a.start : -1, a.path, a.n_tree);
    fresh[i] = from >= 0;
    if (fresh[i]) x[i].load(src + from * a.src_st + (item % kPieces) * (BF16 ? 32 : 64));
    else x[i].clear();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
#pragma unroll
    for (int e = 0; e < 16; e += 2) top = fmaxf(top, fmaxf(fabsf(x[i].at(e)), fabsf(x[i].at(e + 1))));       // a NaN is no maximum
  top = block_max(top, part[0]);
  const bool infinite = top == INFINITY;          // rare: the largest finite magnitude, and infinities at the end of the range
  if (__builtin_expect(infinite, 0)) {
    top = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float v = fabsf(x[i].at(e));
        top = v < INFINITY ? fmaxf(top, v) : top;
      }
    top = block_max(top, part[1]);
  }
  const float scale = fmaxf(quant_scale(top), old_scale);
  const float inv = 1.0f / scale;                 // exact for a power of two
  if (threadIdx.x == 0) *scale_at = scale;
  if (has_older && scale != old_scale) {
    // the older rows of the block under their new scale
    const float ratio = old_scale * inv;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int item = i * kThreads + threadIdx.x;
      const int row = item / kPieces;
      if (row >= rows || pos0 + row >= a.start) continue;
      uintx4* at = reinterpret_cast<uintx4*>(cache + static_cast<int64_t>(pos0 + row) * a.cache_sl + (item % kPieces) * 16);
      uintx4 w = *at;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], true);
        w[e] = encode4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
      }
      *at = w;
    }
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (!fresh[i]) continue;
    const int item = i * kThreads + threadIdx.x;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      v[e] = x[i].at(e) * inv;
      if (__builtin_expect(infinite, 0) && fabsf(v[e]) == INFINITY) v[e] = copysignf(448.f, v[e]);
    }
    uintx4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = encode4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
    *reinterpret_cast<uintx4*>(cache + static_cast<int64_t>(pos0 + item / kPieces) * a.cache_sl + (item % kPieces) * 16) = w;
  }
}

constexpr int kReadItems = 2;

// pieces of 16 values of rows start .. start + n, one after the other
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(QuantRead a) {
  constexpr int kPieces = D / 16;
  const int lh = blockIdx.y;
  const int layer = lh / a.n_kv_heads, g = lh - layer * a.n_kv_heads;
  const bool is_v = blockIdx.z != 0;
  const unsigned char* cache = static_cast<const unsigned char*>(is_v ? a.v_cache : a.k_cache) + layer * a.cache_sy + g * a.cache_sh;
  unsigned char* dst = static_cast<unsigned char*>(is_v ? a.v_dst : a.k_dst) + layer * a.dst_sy + g * a.dst_sh;
  const float* scale = (is_v ? a.v_scale : a.k_scale) + layer * a.scale_sy + g * a.scale_sh;
  uintx4 w[kReadItems];
  float s[kReadItems];
#pragma unroll
  for (int i = 0; i < kReadItems; ++i) {
    const int64_t item = (static_cast<int64_t>(blockIdx.x) * kReadItems + i) * kThreads + threadIdx.x;
    const int row = static_cast<int>(item / kPieces);
    if (row >= a.n_tokens) continue;
    const int pos = a.start + row;
    w[i] = *reinterpret_cast<const uintx4*>(cache + static_cast<int64_t>(pos) * a.cache_sl + (item % kPieces) * 16);
    s[i] = scale[pos >> a.block_log2];
  }
#pragma unroll
  for (int i = 0; i < kReadItems; ++i) {
    const int64_t item = (static_cast<int64_t>(blockIdx.x) * kReadItems + i) * kThreads + threadIdx.x;
    const int row = static_cast<int>(item / kPieces);
    if (row >= a.n_tokens) continue;
    float v[16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][e], true);
      v[4 * e] = lo[0] * s[i], v[4 * e + 1] = lo[1] * s[i], v[4 * e + 2] = hi[0] * s[i], v[4 * e + 3] = hi[1] * s[i];
    }
    uintx4* to = reinterpret_cast<uintx4*>(dst + row * a.dst_st + (item % kPieces) * (BF16 ? 32 : 64));
    if constexpr (BF16) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uintx4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const floatx2 f = {v[8 * h + 2 * e], v[8 * h + 2 * e + 1]};
          o[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
        }
        to[h] = o;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h)
        to[h] = uintx4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
    }
  }
}

template <int D, bool BF16>
hipError_t launch_write(const QuantWrite& a, dim3 grid, hipStream_t stream) {
  switch (((D / 16) << a.block_log2) / kThreads) {
    case 0:
    case 1: return launch_kernel(quant_write_kernel<D, BF16, 1>, grid, dim3(kThreads), 0, stream, a);
    case 2: return launch_kernel(quant_write_kernel<D, BF16, 2>, grid, dim3(kThreads), 0, stream, a);
    default: return launch_kernel(quant_write_kernel<D, BF16, 4>, grid, dim3(kThreads), 0, stream, a);
  }
}

}  // namespace

hipError_t launch_quant_write(const QuantWrite& a, hipStream_t stream) {
  if (a.n_tokens <= 0) return hipSuccess;
  const int blocks = ((a.start + a.n_tokens - 1) >> a.block_log2) - (a.start >> a.block_log2) + 1;
  const dim3 grid(blocks, a.n_layers * a.n_kv_heads, 2);
  if (a.head_dim == 128) return a.bf16 ? launch_write<128, true>(a, grid, stream) : launch_write<128, false>(a, grid, stream);
  return a.bf16 ? launch_write<64, true>(a, grid, stream) : launch_write<64, false>(a, grid, stream);
}

hipError_t launch_quant_read(const QuantRead& a, hipStream_t stream) {
  if (a.n_tokens <= 0) return hipSuccess;
  const int64_t items = static_cast<int64_t>(a.n_tokens) * (a.head_dim / 16);
  const dim3 grid(static_cast<unsigned>((items + kReadItems * kThreads - 1) / (kReadItems * kThreads)), a.n_layers * a.n_kv_heads, 2);
  const dim3 threads(kThreads);
  if (a.head_dim == 128)
    return a.bf16 ? launch_kernel(quant_read_kernel<128, true>, grid, threads, 0, stream, a)
                  : launch_kernel(quant_read_kernel<128, false>, grid, threads, 0, stream, a);
  return a.bf16 ? launch_kernel(quant_read_kernel<64, true>, grid, threads, 0, stream, a)
                : launch_kernel(quant_read_kernel<64, false>, grid, threads, 0, stream, a);
}

}  // namespace specext

// Arguments and small rules of the kernels that fill and read the 8-bit cache (quant_cache.hip).  The rules are callable on the
// host too, so that they can be run there.
#pragma once

#include <cmath>

#include "common.h"

namespace specext {

// Strides in bytes (scales: in floats).
struct QuantWrite {
  const void* k_src;
  const void* v_src;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  const int32_t* path;        // null: row i is source row i; else path[i]
  const int32_t* n_accept;    // null: n_tokens rows; else this many, n_tokens at the most
  int32_t n_tree;             // source rows that path may name
  int32_t n_layers, n_kv_heads, head_dim, bf16;
  int32_t n_tokens, start, block_log2;
  int64_t src_sy, src_sh, src_st, cache_sy, cache_sh, cache_sl, scale_sy, scale_sh;
};

struct QuantRead {
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  void* k_dst;
  void* v_dst;
  int32_t n_layers, n_kv_heads, head_dim, bf16;
  int32_t n_tokens, start, block_log2;
  int64_t cache_sy, cache_sh, cache_sl, dst_sy, dst_sh, dst_st, scale_sy, scale_sh;
};

hipError_t launch_quant_write(const QuantWrite& a, hipStream_t stream);
hipError_t launch_quant_read(const QuantRead& a, hipStream_t stream);

// Smallest power of two s >= 2^-100 with top <= 448 s, for finite top >= 0: 448 = 1.75 x 2^8, so it follows from the exponent and
// from whether the mantissa is above 1.75.
__host__ __device__ __forceinline__ float quant_scale(float top) {
  union { float f; uint32_t u; } v = {top};
  const int e = static_cast<int>(v.u >> 23) - 127 - 8 + ((v.u & 0x7fffffu) > 0x600000u ? 1 : 0);
  v.u = static_cast<uint32_t>((e < -100 ? -100 : e) + 127) << 23;
  return v.f;
}

// The source row of new row i: itself, or the tree node that the path has there; -1 for a row that is not written (i < 0, or no
// node).  No entry of the path behind the accepted ones is read: i is below their count.
__host__ __device__ __forceinline__ int quant_source_row(int i, const int32_t* path, int n_tree) {
  if (i < 0 || !path) return i;
  const int node = path[i];
  return node >= 0 && node < n_tree ? node : -1;
}

}  // namespace specext

// End of the 8-bit prefix kernels whose waves share rows: the partials that GROUPS waves have of a block of 32 rows meet in LDS and
// go out as one.
#pragma once

#include "mfma_util.h"

namespace specext {

// Matrix results before they are read by anything but a matrix instruction.  The compiler keeps the distance that one instruction
// needs from its issue; behind other products, of this wave or its neighbour on the SIMD, one waits in the matrix pipe, and its first
// reader 18 instructions behind it now and then saw the old value (measured: two logits of a lane, in the loop of prefix_quant.hip).
// There the readers are hundreds of cycles away now; where references move and at a kernel's end this waits for them.
template <int N>
__device__ __forceinline__ void settle(floatx16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[i]));
  __builtin_amdgcn_sched_barrier(0);
}

// A wave's O^T accumulators in LDS, four registers of a lane at a time: 16 bytes are four columns of a row.  The lanes' upper half lies
// one such piece further, and so does every four registers twice, so that neighbouring lanes of a row, which read them in turns, and
// the next rows beside them, hit different banks.  (Single words, with bank conflicts in their reads: 16 nodes of 32 heads in 8 groups at
// 2K keys 9.85 us per prefix launch, now 8.8.)
constexpr int kDumpHalf = 33, kDumpStride = 66;          // pieces
template <int D>
__host__ __device__ constexpr int dump_floats() { return D / 8 * kDumpStride * 4; }
// LDS of `waves` (waves x blocks of rows) dumps with their references and sums
template <int D>
__host__ __device__ constexpr int merge_bytes(int waves) { return waves * (dump_floats<D>() + 2 * 32) * 4; }

template <int D>
__device__ __forceinline__ void dump_wave(float* lds, int n_waves, int index, const floatx16 (&acc)[D / 32], float ref, float sum, int lane) {
  floatx4* at = reinterpret_cast<floatx4*>(lds + index * dump_floats<D>()) + (lane & 31) + (lane >> 5) * kDumpHalf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) at[(db * 4 + r) * kDumpStride] = floatx4{acc[db][4 * r], acc[db][4 * r + 1], acc[db][4 * r + 2], acc[db][4 * r + 3]};
  if (lane < 32) reinterpret_cast<floatx2*>(lds + n_waves * dump_floats<D>())[index * 32 + lane] = floatx2{ref, sum};
}

// Rows [0, n_rows) of a block, from dumps index0 + w * index_step of its GROUPS waves; this wave is number `member` of the GROUPS that
// store.  A row is stored whole, by neighbouring lanes (32-byte pieces, as the accumulators hold them, cost the memory several times
// their size): D = 128 as fp16 after the power of two that brings the row's largest element just below 1 (the triple of reference,
// sum and O is rescaled), D = 64 as fp32.
template <int D, int GROUPS>
__device__ __forceinline__ void merge_groups(const float* lds, int n_waves, int index0, int index_step, int member, int n_rows, float* part_o,
                                             float* part_ml, int64_t slot0, int lane) {
  constexpr int kLanes = D / 4;                  // of a row: four columns each
  constexpr int kRows = 64 / kLanes;
  const floatx2* ml = reinterpret_cast<const floatx2*>(lds + n_waves * dump_floats<D>());
  const int q = lane % kLanes;                   // columns 4 q .. 4 q + 3: registers 4 (q / 2) .. + 3 of lanes row + 32 (q & 1)
  const int piece = (q >> 1) * kDumpStride + (q & 1) * kDumpHalf;
#pragma unroll 4
  for (int row0 = member * kRows; row0 < min(n_rows, 32); row0 += GROUPS * kRows) {
    const int row = row0 + lane / kLanes;
    floatx2 part[GROUPS];                        // reference, sum
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < GROUPS; ++w) {
      part[w] = ml[(index0 + w * index_step) * 32 + row];
      top = fmaxf(top, part[w][0]);
    }
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < GROUPS; ++w) {
      const float weight = part[w][1] > 0.f ? fast_exp2(part[w][0] - top) : 0.f;       // a wave without tiles: nothing
      total = fmaf(part[w][1], weight, total);
      const floatx4 x = reinterpret_cast<const floatx4*>(lds + (index0 + w * index_step) * dump_floats<D>())[piece + row];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], weight, o[e]);
    }
    if constexpr (D == 128) {
      float largest = row16_max(fmaxf(fmaxf(fabsf(o[0]), fabsf(o[1])), fmaxf(fabsf(o[2]), fabsf(o[3]))));
      largest = fmaxf(largest, __shfl_xor(largest, 16, 64));
      const int row_exp = largest > 0.f && largest < INFINITY ? __builtin_amdgcn_frexp_expf(largest) : 0;
      const float scale = __builtin_amdgcn_ldexpf(1.0f, -row_exp);
      const floatx2 lo = {o[0] * scale, o[1] * scale}, hi = {o[2] * scale, o[3] * scale};
      const uintx2 h = {__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, halfx2)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, halfx2))};
      if (row < n_rows) {
        __builtin_nontemporal_store(h, reinterpret_cast<uintx2*>(reinterpret_cast<uint16_t*>(part_o) + (slot0 + row) * D + 4 * q));
        if (q == 0) __builtin_nontemporal_store(floatx2{top + static_cast<float>(row_exp), total * scale}, reinterpret_cast<floatx2*>(part_ml + (slot0 + row) * 2));
      }
    } else if (row < n_rows) {
      __builtin_nontemporal_store(o, reinterpret_cast<floatx4*>(part_o + (slot0 + row) * D + 4 * q));
      if (q == 0) __builtin_nontemporal_store(floatx2{top, total}, reinterpret_cast<floatx2*>(part_ml + (slot0 + row) * 2));
    }
  }
}

}  // namespace specext

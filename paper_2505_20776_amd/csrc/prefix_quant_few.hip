// Prefix pass over a target cache held in 8 bits for at most 64 query rows per KV head (decoding, chains, small trees): the cache has
// to be streamed, and nothing else takes long.  The mathematics is that of prefix_quant.hip.
//
// A workgroup is four waves that share the rows and take the 32-key tiles of the split in turns, each through a ring of four tiles
// of its own in LDS, filled by direct loads: 128 KB in flight per compute unit and no barrier before the end.  Nothing is shared, so
// the e4m3 values stay as they are until a wave reads its operands: keys as 16-byte pieces, values through the transposing read of
// bytes, each widened to fp16 in registers, once.  The order of a row's elements within the contraction is the one that the 16-byte
// pieces give, for keys and queries alike; the order of the keys is that of the logits in their accumulator.
//
// With one block of rows the load bounds it: 32 heads in 8 groups, one node, 131035 keys 46.3 us per launch, 5.8 TB/s (37.9 us at
// the 7.08 of a plain read); 16K 11.1 (4.7), 2K 5.3 (0.6): what a launch, the first load and the end take.  With two blocks a wave
// has 32 products per tile behind one another and a softmax for each block, and one wave per SIMD has nothing to put into the gaps:
// 16 nodes 131035 keys 54 to 57; 2K 8.8, of which the end takes 2.8 and the tiles 1.8; 60 nodes of 12 64-wide heads at 1013 keys 5.6.
// Per attention call one node at 2K takes 8.4 us, 16 nodes at 131035 60; with the shared tiles and barriers of prefix_quant.hip they
// were 11.3 and 68.
#include "quant_merge.h"

namespace specext {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((address_space(4))) const float const_float;
typedef __attribute__((ext_vector_type(2))) int intx2;
typedef __attribute__((address_space(3))) intx2 lds_intx2;

constexpr int kWaves = 4;
constexpr int kTile = 32;        // keys
constexpr int kSlots = 4;        // tiles of a wave's ring

template <int D>
__host__ __device__ constexpr int slot_bytes() { return 2 * kTile * D; }        // K and V of a tile
template <int D, int RB>
constexpr int lds_bytes() {
  const int ring = kWaves * kSlots * slot_bytes<D>();
  const int merge = merge_bytes<D>(kWaves * RB);
  return ring > merge ? ring : merge;
}

// at most n vector-memory operations outstanding, n = 28 (the usual case) or even and at most 24
__device__ __forceinline__ void wait_vm(int n) {
  if (__builtin_expect(n == 28, 1)) asm volatile("s_waitcnt vmcnt(28)" ::: "memory");
  else wait_vmcnt_even(n);
}

// eight e4m3 values -> fp16, exactly
__device__ __forceinline__ halfx8 widen8(uint32_t a, uint32_t b) {
  const uintx4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true))};
  return __builtin_bit_cast(halfx8, w);
}

__device__ __forceinline__ halfx8 pack8_f16(const floatx16& v, int first) {
  halfx8 out;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const floatx2 f = {v[first + e], v[first + e + 1]};
    const halfx2 h = __builtin_convertvector(f, halfx2);
    out[e] = h[0];
    out[e + 1] = h[1];
  }
  return out;
}

template <int D, int RB, bool SCORES>
__global__ __launch_bounds__(kWaves * 64) void prefix_quant_few_kernel(uint64_t k_at, uint64_t v_at, uint64_t q_at, int64_t kp_sh, int64_t kp_sl, int L,
                                                                  int keys_per_split, int M, int G, uint64_t k_scale_at, uint64_t v_scale_at,
                                                                  int64_t scale_sh, int block_log2, AttnParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kHalf = kTile * D;               // bytes of a K or V tile
  constexpr int kLoads = kHalf / 1024;           // direct loads of one
  constexpr int kLoadRows = 1024 / D;            // rows of a load
  constexpr int kChunks = D / 16;                // 16-byte pieces of a row
  constexpr int kPieces = D / 32;                // of these, a lane's
  constexpr int kBlocks = D / 32;                // 32-column blocks of the output

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31;
  const int hf = lane >> 5;
  const int split = p.head_fastest ? blockIdx.y : blockIdx.x;
  const int g = p.head_fastest ? blockIdx.x : blockIdx.y;

  const int key_lo = split * keys_per_split;
  const int key_hi = min(L, key_lo + keys_per_split);
  const int n_tiles = (key_hi - key_lo + kTile - 1) / kTile;
  const int n = (n_tiles - wave + kWaves - 1) / kWaves;          // this wave's: wave, wave + 4, ...

  const unsigned char* kbase = in_global<const unsigned char>(k_at) + g * kp_sh;
  const unsigned char* vbase = in_global<const unsigned char>(v_at) + g * kp_sh;

  // ---- loads.  One writes 1 KB of LDS, lane i 16 bytes at 16 i; the swizzle that spares the operand reads bank conflicts is applied
  // to the address that a lane fetches.
  auto k_swizzle = [](int row) { return D == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
  auto v_swizzle = [](int row) { return D == 128 ? (row & 2) | ((row >> 1) & 4) : (row >> 2) & 2; };
  unsigned char* ring = lds + wave * kSlots * slot_bytes<D>();
  const unsigned ring_lds = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)ring));
  const unsigned row_stride = static_cast<unsigned>(kp_sl);
  const int ld_row = lane / kChunks, ld_chunk = lane % kChunks;
  unsigned k_voff[kLoads], v_voff[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int row = u * kLoadRows + ld_row;
    k_voff[u] = row * row_stride + ((ld_chunk ^ k_swizzle(row)) << 4);
    v_voff[u] = row * row_stride + ((ld_chunk ^ v_swizzle(row)) << 4);
  }
  auto tile_key0 = [&](int j) { return key_lo + (wave + kWaves * j) * kTile; };
  auto issue_tile = [&](int j) {
    const int key0 = tile_key0(j);
    const unsigned dst = ring_lds + (j % kSlots) * slot_bytes<D>();
    const unsigned char* kt = kbase + key0 * kp_sl;
    const unsigned char* vt = vbase + key0 * kp_sl;
    if (__builtin_expect(key0 + kTile <= L, 1)) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) load_to_lds_16_stream(dst + u * 1024, k_voff[u], kt);
#pragma unroll
      for (int u = 0; u < kLoads; ++u) load_to_lds_16_stream(dst + kHalf + u * 1024, v_voff[u], vt);
    } else {
      // keys behind the prefix: its last one again, masked below
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int row = u * kLoadRows + ld_row;
        load_to_lds_16_stream(dst + u * 1024, min(row, L - 1 - key0) * row_stride + ((ld_chunk ^ k_swizzle(row)) << 4), kt);
      }
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int row = u * kLoadRows + ld_row;
        load_to_lds_16_stream(dst + kHalf + u * 1024, min(row, L - 1 - key0) * row_stride + ((ld_chunk ^ v_swizzle(row)) << 4), vt);
      }
    }
  };

  // ---- the queries come first and the same way, into the ring's last slots, beside the first tiles
  constexpr int kQRowBytes = D * 2;
  constexpr int kQChunks = D / 8;
  constexpr int kQLoadRows = 1024 / kQRowBytes;
  constexpr int kQLoads = 32 / kQLoadRows;       // of a row block
  constexpr int kQSlots = RB * 32 * kQRowBytes / slot_bytes<D>();       // slots that they take
  static_assert(kQSlots < kSlots, "a slot for the first tile");
  auto q_swizzle = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  const unsigned q_lds = ring_lds + (kSlots - kQSlots) * slot_bytes<D>();
  if (n > 0) {
    const float inv_g = 1.0f / static_cast<float>(G);
    const unsigned q_st = static_cast<unsigned>(p.q_st) * 2u, q_sh = static_cast<unsigned>(p.q_sh) * 2u;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int u = 0; u < kQLoads; ++u) {
        const int row = u * kQLoadRows + lane / kQChunks;
        const int m = min(32 * rb + row, M - 1);             // padding rows repeat the last real row (never stored)
        const int t = static_cast<int>((static_cast<float>(m) + 0.5f) * inv_g);       // m / G, exact for m < 2^20
        const int h = g * G + (m - t * G);
        load_to_lds_16(q_lds + (rb * kQLoads + u) * 1024, t * q_st + h * q_sh + (((lane % kQChunks) ^ q_swizzle(row)) << 4),
                       in_global<const unsigned char>(q_at));
      }
#pragma unroll
    for (int j = 0; j < kSlots - kQSlots; ++j)
      if (j < n) issue_tile(j);
  }

  floatx16 acc_o[RB][kBlocks];
  halfx8 qf[RB][2 * kPieces];
  float ref[RB], run_sum[RB], c[RB];       // base-2 reference, the values' scale included; lane-partial sum; factor of the logits
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    ref[rb] = -INFINITY;
    run_sum[rb] = 0.f;
    c[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc_o[rb][db][r] = 0.f;
  }
  const const_float* k_scale = (const const_float*)k_scale_at + g * scale_sh;
  const const_float* v_scale = (const const_float*)v_scale_at + g * scale_sh;

  // operand reads: piece i of key c32 is chunk 2 i + hf of its row; values of 8 keys and 16 columns per group of 16 lanes
  unsigned k_rd[kPieces], v_rd[kBlocks];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) k_rd[i] = ring_lds + c32 * D + (((2 * i + hf) ^ k_swizzle(c32)) << 4);
  {
    const int li = lane & 15, half16 = (lane >> 4) & 1;
    const int e = li >> 1;                       // element of the contraction that this lane's row is
    const int row = 8 * (e >> 2) + 4 * hf + (e & 3);         // + 16 jj: the swizzle is that of these rows too
#pragma unroll
    for (int db = 0; db < kBlocks; ++db) v_rd[db] = ring_lds + kHalf + row * D + (((2 * db + half16) ^ v_swizzle(row)) << 4) + ((li & 1) << 3);
  }

  if (n > 0) {
    // queries: moved to 2^8 at the most by a power of two, as fp16
    {
      const int younger = 2 * kLoads * min(n, kSlots - kQSlots);
      wait_vm(younger);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        uintx4 w[2 * kPieces];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i) {
          const int chunk = 2 * (2 * (i >> 1) + hf) + (i & 1);
          w[i] = *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(q_lds + rb * 32 * kQRowBytes + c32 * kQRowBytes + ((chunk ^ q_swizzle(c32)) << 4)));
        }
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i][e] << 16)), fabsf(__uint_as_float(w[i][e] & 0xffff0000u))));
        top = halves_max(top);
        const int shift = top > 0.f && top < INFINITY ? 8 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const floatx2 f = {__builtin_amdgcn_ldexpf(__uint_as_float(w[i][e] << 16), shift),
                               __builtin_amdgcn_ldexpf(__uint_as_float(w[i][e] & 0xffff0000u), shift)};
            const halfx2 hh = __builtin_convertvector(f, halfx2);
            qf[rb][i][2 * e] = hh[0];
            qf[rb][i][2 * e + 1] = hh[1];
          }
        c[rb] = __builtin_amdgcn_ldexpf(p.scale_log2, -shift);
      }
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the queries are in registers: their slots are free
#pragma unroll
      for (int j = kSlots - kQSlots; j < kSlots; ++j)
        if (j < n) issue_tile(j);
      __builtin_amdgcn_sched_barrier(0);
    }

    for (int j = 0; j < n; ++j) {
      const int key0 = tile_key0(j);
      const unsigned slot = (j % kSlots) * slot_bytes<D>();
      const int block = key0 >> block_log2;
      const float sk = k_scale[block], sv = v_scale[block];
      // K of this tile: younger are its V and the tiles behind it, up to three
      const int behind = min(n - 1 - j, kSlots - 1);
      wait_vm(kLoads * (1 + 2 * behind));
      halfx8 kf[2 * kPieces];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const uintx4 w = *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(k_rd[i] + slot));
        kf[2 * i] = widen8(w[0], w[1]);
        kf[2 * i + 1] = widen8(w[2], w[3]);
      }
      floatx16 s[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        s[rb] = floatx16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2 * kPieces; ++i)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i], qf[rb][i], s[rb], 0, 0, 0);
      // (the products stay here, far in front of the first reader of their results: see settle())
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(s[rb]));
      // V: widened while the logits come out of the matrix pipe
      wait_vm(kLoads * 2 * behind);
      halfx8 vf[2][kBlocks];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int db = 0; db < kBlocks; ++db) {
          const intx2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_intx2*)static_cast<uintptr_t>(v_rd[db] + slot + 16 * jj * D));
          vf[jj][db] = widen8(w[0], w[1]);
        }
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // this slot has been read: the tile four behind takes it
      if (j + kSlots < n) issue_tile(j + kSlots);
      __builtin_amdgcn_sched_barrier(0);

      const float lsv = __builtin_amdgcn_logf(sv);
      const float inv_sv = __builtin_amdgcn_rcpf(sv);
      // register r of s holds key key0 + 8 (r / 4) + 4 hf + r % 4
      if (__builtin_expect(key0 + kTile > key_hi, 0)) {
        const int left = key_hi - key0 - 4 * hf;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (8 * (r >> 2) + (r & 3) >= left) s[rb][r] = -INFINITY;
      }
      float top[RB];
      bool grow = false;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        top[rb] = fmaxf(s[rb][0], s[rb][1]);
#pragma unroll
        for (int r = 2; r < 16; r += 2) top[rb] = fmaxf(top[rb], fmaxf(s[rb][r], s[rb][r + 1]));
        top[rb] = fmaf(top[rb], c[rb] * sk, lsv);
        grow |= top[rb] > ref[rb] + kLazyLog2;
      }
      if (__builtin_expect(__any(grow), 0)) {      // some row of this wave outgrew its reference: move every reference up
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float new_ref = fmaxf(ref[rb], halves_max(top[rb]));
          const float alpha = fast_exp2(ref[rb] - new_ref);             // 0 on the first tile
          ref[rb] = new_ref;
          run_sum[rb] *= alpha;
#pragma unroll
          for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc_o[rb][db][r] *= alpha;
        }
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float ct = c[rb] * sk, shift = lsv - ref[rb];
        float part = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[rb][r] = fast_exp2(fmaf(s[rb][r], ct, shift));
          part += s[rb][r];
        }
        part *= inv_sv;
        run_sum[rb] += part;
        if (SCORES) {
          // every lane stores: the two lanes of a row hold the same pair, and so do padding rows
          unsigned char* block_at = reinterpret_cast<unsigned char*>(p.chunk_part) + (static_cast<int64_t>(g) * p.n_sub + key0 / kTile) * M * 8;
          *reinterpret_cast<floatx2*>(block_at + static_cast<unsigned>(min(32 * rb + c32, M - 1)) * 8u) = floatx2{halves_sum(part), ref[rb]};
        }
        const halfx8 p0 = pack8_f16(s[rb], 0), p1 = pack8_f16(s[rb], 8);
#pragma unroll
        for (int jj = 0; jj < 2; ++jj)
#pragma unroll
          for (int db = 0; db < kBlocks; ++db) acc_o[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[jj][db], jj ? p1 : p0, acc_o[rb][db], 0, 0, 0);
      }
    }
  }

  // ---- the four waves' partials of a block of rows meet in LDS
  float* dump = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    settle(acc_o[rb]);
    run_sum[rb] = halves_sum(run_sum[rb]);
  }
  __syncthreads();                                   // every wave is done with its ring
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) dump_wave<D>(dump, kWaves * RB, wave * RB + rb, acc_o[rb], ref[rb], run_sum[rb], lane);
  __syncthreads();
  const int64_t slot0 = static_cast<int64_t>(split) * p.Hq * p.T + g * M;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
    merge_groups<D, kWaves>(dump, kWaves * RB, rb, RB, wave, M - 32 * rb, p.part_o, p.part_ml, slot0 + 32 * rb, lane);
}

template <int D, int RB, bool SCORES>
hipError_t launch_one(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  auto kernel = prefix_quant_few_kernel<D, RB, SCORES>;
  constexpr int kLdsBytes = lds_bytes<D, RB>();
  static_assert(kLdsBytes <= 160 * 1024, "the rings fit the LDS");
  if (kLdsBytes > 64 * 1024) {
    // more than the default 64 KB of dynamic LDS: raise the cap once per device
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
      if (e != hipSuccess) return e;
      attr_set[dev].store(true, std::memory_order_release);
    }
  }
  dim3 grid(p.head_fastest ? p.Hkv : p.S, p.head_fastest ? p.S : p.Hkv);
  return launch_kernel(kernel, grid, dim3(kWaves * 64), kLdsBytes, stream, address_of(p.kp), address_of(p.vp), address_of(p.q), p.kp_sh, p.kp_sl,
                       p.L, p.keys_per_split, p.M, p.G, address_of(s.k), address_of(s.v), s.sh, s.block_log2, p);
}

template <int D, bool SCORES>
hipError_t launch_rows(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  return p.M <= 32 ? launch_one<D, 1, SCORES>(p, s, stream) : launch_one<D, 2, SCORES>(p, s, stream);
}

}  // namespace

hipError_t launch_prefix_quant_few(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  if (p.d == 128) return p.want_scores ? launch_rows<128, true>(p, s, stream) : launch_rows<128, false>(p, s, stream);
  return p.want_scores ? launch_rows<64, true>(p, s, stream) : launch_rows<64, false>(p, s, stream);
}

}  // namespace specext

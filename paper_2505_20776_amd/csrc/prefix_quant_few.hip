// Prefix pass over a target cache held in 8 bits for at most 64 query rows per KV head (decoding, chains, small trees): the cache has
// to be streamed, and nothing else takes long.  The mathematics is that of prefix_quant.hip.
//
// A workgroup is four groups that take the 32-key tiles of the split in turns, each through a ring of four tiles of its own in LDS,
// filled by direct loads: 128 KB on its way per compute unit.  A group is one wave where there are at most 32 rows; then nothing is
// shared and there is no barrier before the end.  For up to 64 rows it is two waves, with 32 rows each, over one ring: a barrier per
// tile, and the second product of a tile behind the next one's barrier, from registers, while K comes from LDS.  The e4m3 values stay
// as they are until a wave reads its operands: keys as 16-byte pieces, values through the transposing read of bytes, each widened to
// fp16 in registers.  The order of a row's elements within the contraction is the one that the 16-byte pieces give, for keys and
// queries alike; the order of the keys is that of the logits in their accumulator.
//
// One block of rows is bound by the load: 32 heads in 8 groups, one node, 131035 keys 46.3 us per launch, 5.8 TB/s (37.9 us at the 7.08
// of a plain read); 16K 11.1 (4.7), 2K 5.3 (0.6): what a launch, the first load and the end take.  Two blocks, 16 nodes: 131035 keys
// 58.5 us, 4.6 TB/s and 0.59 PFLOP/s, 8K 10.7, 2K 8.0; 60 nodes of 12 64-wide heads, 1013 keys 5.5.  One wave with both blocks, which
// widens and reads half as much but has its SIMD to itself, so that nothing fills the gaps between its products: 57.9, 11.4, 8.8 and
// 5.7.  (A ring of five tiles: 62 at 131035.)  Per attention call one node at 2K takes 8.5 us, 16 nodes 11.5; one node was 11.3 with
// the tiles widened once for all waves, as in prefix_quant.hip.
#include "quant_merge.h"

namespace specext {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((address_space(4))) const float const_float;
typedef __attribute__((ext_vector_type(2))) int intx2;
typedef __attribute__((address_space(3))) intx2 lds_intx2;

constexpr int kGroups = 4;       // of keys: a wave for one block of rows, two for two
constexpr int kTile = 32;        // keys
constexpr int kSlots = 4;        // tiles of a group's ring

template <int D>
__host__ __device__ constexpr int slot_bytes() { return 2 * kTile * D; }        // K and V of a tile
template <int D, int R>
constexpr int lds_bytes() {
  const int ring = kGroups * kSlots * slot_bytes<D>();
  const int merge = merge_bytes<D>(kGroups * R);
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

template <int D, int R, bool SCORES>
__global__ __launch_bounds__(kGroups * R * 64) void prefix_quant_few_kernel(uint64_t k_at, uint64_t v_at, uint64_t q_at, int64_t kp_sh, int64_t kp_sl, int L,
                                                                  int keys_per_split, int M, int G, uint64_t k_scale_at, uint64_t v_scale_at,
                                                                  int64_t scale_sh, int block_log2, AttnParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kHalf = kTile * D;               // bytes of a K or V tile
  constexpr int kLoads = kHalf / 1024;           // direct loads of one
  constexpr int kLoadRows = 1024 / D;            // rows of a load
  constexpr int kChunks = D / 16;                // 16-byte pieces of a row
  constexpr int kTileLoads = 2 * kLoads / R;     // of a tile, a wave's
  constexpr int kPieces = D / 32;                // of these, a lane's
  constexpr int kBlocks = D / 32;                // 32-column blocks of the output

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / R, r_block = wave % R;
  const int c32 = lane & 31;
  const int hf = lane >> 5;
  const int split = p.head_fastest ? blockIdx.y : blockIdx.x;
  const int g = p.head_fastest ? blockIdx.x : blockIdx.y;

  const int key_lo = split * keys_per_split;
  const int key_hi = min(L, key_lo + keys_per_split);
  const int n_tiles = (key_hi - key_lo + kTile - 1) / kTile;
  const int n = (n_tiles - kg + kGroups - 1) / kGroups;          // this group's: kg, kg + 4, ...

  const unsigned char* kbase = in_global<const unsigned char>(k_at) + g * kp_sh;
  const unsigned char* vbase = in_global<const unsigned char>(v_at) + g * kp_sh;

  // ---- loads.  One writes 1 KB of LDS, lane i 16 bytes at 16 i; the swizzle that spares the operand reads bank conflicts is applied
  // to the address that a lane fetches.
  auto k_swizzle = [](int row) { return D == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
  auto v_swizzle = [](int row) { return D == 128 ? (row & 2) | ((row >> 1) & 4) : (row >> 2) & 2; };
  unsigned char* ring = lds + kg * kSlots * slot_bytes<D>();
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
  auto tile_key0 = [&](int j) { return key_lo + (kg + kGroups * j) * kTile; };
  // (of two waves the one brings K, the other V)
  auto issue_rows = [&](int j, bool is_v) __attribute__((always_inline)) {
    const int key0 = tile_key0(j);
    const unsigned dst = ring_lds + (j % kSlots) * slot_bytes<D>() + (is_v ? kHalf : 0);
    const unsigned char* at = (is_v ? vbase : kbase) + key0 * kp_sl;
    if (__builtin_expect(key0 + kTile <= L, 1)) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) load_to_lds_16_stream(dst + u * 1024, is_v ? v_voff[u] : k_voff[u], at);
    } else {
      // keys behind the prefix: its last one again, masked below
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int row = u * kLoadRows + ld_row;
        load_to_lds_16_stream(dst + u * 1024, min(row, L - 1 - key0) * row_stride + ((ld_chunk ^ (is_v ? v_swizzle(row) : k_swizzle(row))) << 4), at);
      }
    }
  };
  auto issue_tile = [&](int j) __attribute__((always_inline)) {
    if (R == 1 || r_block == 0) issue_rows(j, false);
    if (R == 1 || r_block == 1) issue_rows(j, true);
  };

  // ---- the queries come first and the same way, into the ring's last slots, beside the first tiles
  constexpr int kQRowBytes = D * 2;
  constexpr int kQChunks = D / 8;
  constexpr int kQLoadRows = 1024 / kQRowBytes;
  constexpr int kQLoads = 32 / kQLoadRows;       // of a row block
  constexpr int kQSlots = R * 32 * kQRowBytes / slot_bytes<D>();        // slots that they take
  static_assert(kQSlots < kSlots, "a slot for the first tile");
  auto q_swizzle = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  const unsigned q_lds = ring_lds + (kSlots - kQSlots) * slot_bytes<D>() + r_block * 32 * kQRowBytes;
  if (n > 0) {
    const float inv_g = 1.0f / static_cast<float>(G);
    const unsigned q_st = static_cast<unsigned>(p.q_st) * 2u, q_sh = static_cast<unsigned>(p.q_sh) * 2u;
#pragma unroll
    for (int u = 0; u < kQLoads; ++u) {
      const int row = u * kQLoadRows + lane / kQChunks;
      const int m = min(32 * r_block + row, M - 1);          // padding rows repeat the last real row (never stored)
      const int t = static_cast<int>((static_cast<float>(m) + 0.5f) * inv_g);       // m / G, exact for m < 2^20
      const int h = g * G + (m - t * G);
      load_to_lds_16(q_lds + u * 1024, t * q_st + h * q_sh + (((lane % kQChunks) ^ q_swizzle(row)) << 4), in_global<const unsigned char>(q_at));
    }
#pragma unroll
    for (int j = 0; j < kSlots - kQSlots; ++j)
      if (j < n) issue_tile(j);
  }

  floatx16 acc_o[kBlocks];
#pragma unroll
  for (int db = 0; db < kBlocks; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc_o[db][r] = 0.f;
  halfx8 qf[2 * kPieces];
  float ref = -INFINITY, run_sum = 0.f, c = 0.f;       // base-2 reference, the values' scale included; lane-partial sum; factor of the logits
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
    wait_vm(kTileLoads * min(n, kSlots - kQSlots));
    uintx4 w[2 * kPieces];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * kPieces; ++i) {
      const int chunk = 2 * (2 * (i >> 1) + hf) + (i & 1);
      w[i] = *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(q_lds + c32 * kQRowBytes + ((chunk ^ q_swizzle(c32)) << 4)));
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
        qf[i][2 * e] = hh[0];
        qf[i][2 * e + 1] = hh[1];
      }
    c = __builtin_amdgcn_ldexpf(p.scale_log2, -shift);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the queries are in registers: their slots are free
    if (R == 1) {
#pragma unroll
      for (int j = kSlots - kQSlots; j < kSlots; ++j)
        if (j < n) issue_tile(j);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  halfx8 p0 = {}, p1 = {}, vf[2][kBlocks] = {};
  auto second_product = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[jj][db], jj ? p1 : p0, acc_o[db], 0, 0, 0);
  };

  // One wave per group: no barrier, four tiles on their way.  Two: both have to see what both have brought, and a slot is free when both
  // have read it.  The barrier of tile j says both: tile j is there, and the slot of tile j - 1 (for j = 0 those of the queries) can
  // take tile j + 3.
  const int rounds = R == 1 ? n : (n_tiles + kGroups - 1) / kGroups;       // the same for all waves where there is a barrier
  for (int j = 0; j < rounds; ++j) {
    const int behind = R == 1 ? min(n - 1 - j, kSlots - 1) : max(min(n - 1 - j, j == 0 ? 1 : kSlots - 2), 0);
    if (R > 1) {
      wait_vm(kTileLoads * behind);
      __builtin_amdgcn_sched_barrier(0);
      lds_barrier();
#pragma unroll
      for (int i = kSlots - kQSlots; i < kSlots; ++i)
        if ((j == 0 || i == kSlots - 1) && j + i < n) issue_tile(j + i);
      __builtin_amdgcn_sched_barrier(0);
      if (j >= n) continue;
    }
    const int key0 = tile_key0(j);
    const unsigned slot = (j % kSlots) * slot_bytes<D>();
    const int block = key0 >> block_log2;
    const float sk = k_scale[block], sv = v_scale[block];
    // K of this tile: younger are its V and the tiles behind it, up to three
    if (R == 1) wait_vm(kLoads * (1 + 2 * behind));
    uintx4 raw[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) raw[i] = *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(k_rd[i] + slot));
    if (R > 1) second_product();                 // of the tile before, from registers, while K comes from LDS
    halfx8 kf[2 * kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      kf[2 * i] = widen8(raw[i][0], raw[i][1]);
      kf[2 * i + 1] = widen8(raw[i][2], raw[i][3]);
    }
    floatx16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2 * kPieces; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i], qf[i], s, 0, 0, 0);
    // (the products stay here, far in front of the first reader of their results: see settle())
    asm volatile("" : "+v"(s));
    // V: widened while the logits come out of the matrix pipe
    if (R == 1) wait_vm(kTileLoads * behind);
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) {
        const intx2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_intx2*)static_cast<uintptr_t>(v_rd[db] + slot + 16 * jj * D));
        vf[jj][db] = widen8(w[0], w[1]);
      }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // this slot has been read
    if (R == 1 && j + kSlots < n) issue_tile(j + kSlots);    // the tile four behind takes it
    __builtin_amdgcn_sched_barrier(0);

    const float lsv = __builtin_amdgcn_logf(sv);
    const float inv_sv = __builtin_amdgcn_rcpf(sv);
    // register r of s holds key key0 + 8 (r / 4) + 4 hf + r % 4
    if (__builtin_expect(key0 + kTile > key_hi, 0)) {
      const int left = key_hi - key0 - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= left) s[r] = -INFINITY;
    }
    const float ct = c * sk;
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) top = fmaxf(top, fmaxf(s[r], s[r + 1]));
    top = fmaf(top, ct, lsv);
    if (__builtin_expect(__any(top > ref + kLazyLog2), 0)) {     // some row of this wave outgrew its reference: move every reference up
      if (R > 1) settle(acc_o);                                  // (the other wave's products may have kept this one's back)
      const float new_ref = fmaxf(ref, halves_max(top));
      const float alpha = fast_exp2(ref - new_ref);              // 0 on the first tile
      ref = new_ref;
      run_sum *= alpha;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc_o[db][r] *= alpha;
    }
    const float shift = lsv - ref;
    float part = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(fmaf(s[r], ct, shift));
      part += s[r];
    }
    part *= inv_sv;
    run_sum += part;
    if (SCORES) {
      // every lane stores: the two lanes of a row hold the same pair, and so do padding rows
      unsigned char* block_at = reinterpret_cast<unsigned char*>(p.chunk_part) + (static_cast<int64_t>(g) * p.n_sub + key0 / kTile) * M * 8;
      *reinterpret_cast<floatx2*>(block_at + static_cast<unsigned>(min(32 * r_block + c32, M - 1)) * 8u) = floatx2{halves_sum(part), ref};
    }
    p0 = pack8_f16(s, 0), p1 = pack8_f16(s, 8);
    if (R == 1) second_product();
  }
  if (R > 1) second_product();

  // ---- the four groups' partials of a block of rows meet in LDS
  float* dump = reinterpret_cast<float*>(lds);
  settle(acc_o);
  run_sum = halves_sum(run_sum);
  __syncthreads();                                   // every wave is done with its ring
  dump_wave<D>(dump, kGroups * R, wave, acc_o, ref, run_sum, lane);
  __syncthreads();
  const int64_t slot0 = static_cast<int64_t>(split) * p.Hq * p.T + g * M + 32 * r_block;
  merge_groups<D, kGroups>(dump, kGroups * R, r_block, R, kg, M - 32 * r_block, p.part_o, p.part_ml, slot0, lane);
}

template <int D, int R, bool SCORES>
hipError_t launch_one(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  auto kernel = prefix_quant_few_kernel<D, R, SCORES>;
  constexpr int kLdsBytes = lds_bytes<D, R>();
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
  return launch_kernel(kernel, grid, dim3(kGroups * R * 64), kLdsBytes, stream, address_of(p.kp), address_of(p.vp), address_of(p.q), p.kp_sh, p.kp_sl,
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

// Prefix pass of Hybrid Tree Attention (SpecExtend Sec. 3.1) over a target cache held in 8 bits: e4m3 keys and values with one
// scale per block of 32, 64 or 128 tokens and KV head, streamed once from HBM, on the gfx950 matrix cores.
//
//   s[row][j] = c q[row] . (sk k8[j])        o[row] = sum_j 2^s[row][j] (sv v8[j]),   c = softmax scale x log2 e
//
// A tile is 32 keys, so it has one sk and one sv.  sk multiplies the logits of the tile, where a factor is there anyway.  sv goes
// into the exponent: p = 2^(s + log2 sv - ref), so the reference follows the size of what is summed, p stays below 2^kLazyLog2
// whatever the scales, and the row sum takes the tile's p divided by sv.  No scale ever multiplies a key or a value.
//
// Matrix cores: v_mfma_f32_32x32x16_f16.  e4m3 values are fp16 values; a row of bf16 queries is one of fp16 values once its
// largest element has been moved to 2^8 by a power of two (elements below 2^-22 of it lose bits, by 2^-33 of it at most); p has
// 11 bits in fp16 where bf16 would keep 8.  (The 8-bit matrix instructions would take k8 as it is, but align the products of a
// dot product to the largest one and drop what falls below: up to 1.5e-4 of the sum of magnitudes.)
//
// A workgroup is R x KG waves: R blocks of 32 query rows of one KV head, KG groups that take the tiles of the split in turns.
// Every thread brings 16 bytes of e4m3 at a time through registers, PF stages ahead, turns them into fp16 once for the whole
// workgroup and stores them to one of two LDS buffers, while the waves compute on the other: one barrier per stage of KG tiles.
// From there on the tile is that of the bf16 kernels: S^T = K Q^T and O^T += V^T P^T with a lane owning one query row in both
// products, V through the transposing LDS read, P straight from the accumulator registers.
#include "mfma_util.h"

namespace specext {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((address_space(4))) const float const_float;

constexpr int kTile = 32;      // keys per tile

template <int D>
__host__ __device__ constexpr int tile_bytes() { return kTile * D * 2; }      // K or V of a tile as fp16
template <int D, int R, int KG>
constexpr int lds_bytes() {
  const int buffers = 2 * KG * 2 * tile_bytes<D>();
  const int merge = KG > 1 ? R * KG * (D * kTile * 4 + 2 * 32 * 4) : 0;
  return buffers > merge ? buffers : merge;
}

// four e4m3 values -> fp16, exactly
__device__ __forceinline__ void widen4(uint32_t w, uint32_t* out) {
  out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
  out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
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

template <int D, int R, int KG, int PF, bool SCORES>
__global__ __launch_bounds__(R * KG * 64) void prefix_quant_kernel(uint64_t k_at, uint64_t v_at, uint64_t q_at, int64_t kp_sh, int64_t kp_sl, int L,
                                                                 int keys_per_split, int M, int G, uint64_t k_scale_at, uint64_t v_scale_at,
                                                                 int64_t scale_sh, int block_log2, AttnParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kRowBytes = D * 2;
  constexpr int kTileBytes = tile_bytes<D>();
  constexpr int kSteps = D / 16;                 // 16-wide contraction steps of the first product
  constexpr int kBlocks = D / 32;                // 32-column blocks of the output
  constexpr int kPieces = D / 16;                // 1 KB of e4m3 each, of a tile's K and then of its V
  constexpr int kPiecesPerWave = (kPieces + R - 1) / R;
  constexpr int kPieceRows = 1024 / D;
  constexpr int kLanesPerRow = D / 16;
  static_assert(PF % 2 == 0, "the LDS buffer of a stage follows from its place in the unrolled loop");

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / R, r_block = wave % R;
  const int c32 = lane & 31;
  const int hf = lane >> 5;
  const int split = p.head_fastest ? blockIdx.y : blockIdx.x;
  const int g = p.head_fastest ? blockIdx.x : blockIdx.y;
  const int row0 = blockIdx.z * (R * 32) + r_block * 32;
  const bool wave_live = row0 < M;               // a wave of padding rows loads and converts its share, no more

  const int key_lo = split * keys_per_split;
  const int key_hi = min(L, key_lo + keys_per_split);
  const int n_tiles = (key_hi - key_lo + kTile - 1) / kTile;
  const int n_stages = (n_tiles + KG - 1) / KG;

  // ---- loads: this thread's 16-byte pieces of the tile of its key group
  const unsigned char* kbase = in_global<const unsigned char>(k_at) + g * kp_sh;
  const unsigned char* vbase = in_global<const unsigned char>(v_at) + g * kp_sh;
  uintx4 raw[PF][kPiecesPerWave];
  auto load_stage = [&](auto slot_c, int t) __attribute__((always_inline)) {
    constexpr int slot = decltype(slot_c)::value;
    const int key0 = key_lo + (t * KG + kg) * kTile;
#pragma unroll
    for (int i = 0; i < kPiecesPerWave; ++i) {
      const int piece = i * R + r_block;
      if (kPieces < R && piece >= kPieces) continue;
      const bool is_v = piece >= kPieces / 2;
      const int row = (is_v ? piece - kPieces / 2 : piece) * kPieceRows + lane / kLanesPerRow;
      // keys behind the prefix: its last one again, masked below
      const int64_t off = static_cast<int64_t>(min(key0 + row, L - 1)) * kp_sl + (lane % kLanesPerRow) * 16;
      raw[slot][i] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>((is_v ? vbase : kbase) + off));
    }
  };
  // ---- LDS: per buffer and key group a K and a V tile of 32 rows.  The 16-byte chunks of a row are XOR-swizzled so that the
  // operand reads are free of bank conflicts.
  auto k_swizzle = [](int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); };
  auto v_swizzle = [](int row) { return D == 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); };
  auto store_stage = [&](auto slot_c, auto buf_c) __attribute__((always_inline)) {
    constexpr int slot = decltype(slot_c)::value;
    constexpr int buf = decltype(buf_c)::value;
#pragma unroll
    for (int i = 0; i < kPiecesPerWave; ++i) {
      const int piece = i * R + r_block;
      if (kPieces < R && piece >= kPieces) continue;
      const bool is_v = piece >= kPieces / 2;
      const int row = (is_v ? piece - kPieces / 2 : piece) * kPieceRows + lane / kLanesPerRow;
      const int chunk = 2 * (lane % kLanesPerRow);
      const int swizzle = is_v ? v_swizzle(row) : k_swizzle(row);
      unsigned char* dst = lds + (buf * KG + kg) * 2 * kTileBytes + (is_v ? kTileBytes : 0) + row * kRowBytes;
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) widen4(raw[slot][i][e], h + 2 * e);
      *reinterpret_cast<uintx4*>(dst + ((chunk ^ swizzle) << 4)) = uintx4{h[0], h[1], h[2], h[3]};
      *reinterpret_cast<uintx4*>(dst + (((chunk + 1) ^ swizzle) << 4)) = uintx4{h[4], h[5], h[6], h[7]};
    }
  };
  static_for<0, PF>([&](auto u_c) {
    if (decltype(u_c)::value < n_stages) load_stage(u_c, decltype(u_c)::value);
  });

  // ---- queries: B operand of S^T (lane = row c32, 8 consecutive d per step), moved to 2^8 at the most
  halfx8 qf[kSteps];
  float c;
  {
    const int m = min(row0 + c32, M - 1);        // padding rows repeat the last real row (never stored)
    const int t = m / G;
    const int h = g * G + (m - t * G);
    const unsigned char* src = in_global<const unsigned char>(q_at) + (t * p.q_st + h * p.q_sh + 8 * hf) * 2;
    uintx4 w[kSteps];
    float top = 0.f;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) w[ks] = *reinterpret_cast<const uintx4*>(src + 32 * ks);
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[ks][e] << 16)), fabsf(__uint_as_float(w[ks][e] & 0xffff0000u))));
    top = halves_max(top);
    const int shift = top > 0.f && top < INFINITY ? 8 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const floatx2 f = {__builtin_amdgcn_ldexpf(__uint_as_float(w[ks][e] << 16), shift),
                           __builtin_amdgcn_ldexpf(__uint_as_float(w[ks][e] & 0xffff0000u), shift)};
        const halfx2 hh = __builtin_convertvector(f, halfx2);
        qf[ks][2 * e] = hh[0];
        qf[ks][2 * e + 1] = hh[1];
      }
    c = __builtin_amdgcn_ldexpf(p.scale_log2, -shift);
  }

  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)lds)) + kg * 2 * kTileBytes;
  unsigned k_addr[kSteps], v_addr[kBlocks];
#pragma unroll
  for (int ks = 0; ks < kSteps; ++ks) k_addr[ks] = lds0 + c32 * kRowBytes + (((2 * ks + hf) ^ k_swizzle(c32)) << 4);
  {
    // transposing read: a group of 16 lanes reads 4 keys x 16 columns
    const int li = lane & 15, half16 = (lane >> 4) & 1;
    const int row = 4 * hf + (li >> 2);          // + 16 jj (+ 8): the swizzle is that of these rows too
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
      v_addr[db] = lds0 + kTileBytes + row * kRowBytes + (((4 * db + 2 * half16 + ((li & 3) >> 1)) ^ v_swizzle(row)) << 4) + ((li & 1) << 3);
  }

  const const_float* k_scale = (const const_float*)k_scale_at + g * scale_sh;
  const const_float* v_scale = (const const_float*)v_scale_at + g * scale_sh;

  floatx16 acc_o[kBlocks];
#pragma unroll
  for (int db = 0; db < kBlocks; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc_o[db][r] = 0.f;
  float ref = -INFINITY;       // base-2 reference of the row's exponentials, the values' scale included
  float run_sum = 0.f;         // lane-partial row sum
  const int64_t score_step = static_cast<int64_t>(M) * 8;
  unsigned char* score_base = nullptr;
  const unsigned score_off = static_cast<unsigned>(min(row0 + c32, M - 1)) * 8u;
  if (SCORES) score_base = reinterpret_cast<unsigned char*>(p.chunk_part) + (static_cast<int64_t>(g) * p.n_sub + key_lo / kTile) * score_step;

  auto compute = [&](int j, auto buf_c) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value * KG * 2 * kTileBytes;
    const int key0 = key_lo + j * kTile;
    const float sk = k_scale[key0 >> block_log2];
    const float sv = v_scale[key0 >> block_log2];
    floatx16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
      const uintx4 kw = *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(k_addr[ks] + buf));
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, kw), qf[ks], s, 0, 0, 0);
    }
    halfx8 vf[kBlocks][2];
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const unsigned at = v_addr[db] + buf + 16 * jj * kRowBytes;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)static_cast<uintptr_t>(at));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)static_cast<uintptr_t>(at + 8 * kRowBytes));
        vf[db][jj] = __builtin_bit_cast(halfx8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    // register r of s holds key key0 + 8 (r / 4) + 4 hf + r % 4
    if (__builtin_expect(key0 + kTile > key_hi, 0)) {
      const int left = key_hi - key0 - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= left) s[r] = -INFINITY;
    }
    const float ct = c * sk;
    const float lsv = __builtin_amdgcn_logf(sv);
    const float inv_sv = __builtin_amdgcn_rcpf(sv);
    float mx = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) mx = fmaxf(mx, fmaxf(s[r], s[r + 1]));
    mx = fmaf(mx, ct, lsv);
    if (__builtin_expect(__any(mx > ref + kLazyLog2), 0)) {     // some row of this wave outgrew its reference: move every reference up
      const float new_ref = fmaxf(ref, halves_max(mx));
      const float alpha = fast_exp2(ref - new_ref);             // 0 on the first tile
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
    // every lane stores: the two lanes of a row hold the same pair, and so do padding rows
    if (SCORES) *reinterpret_cast<floatx2*>(score_base + j * score_step + score_off) = floatx2{halves_sum(part), ref};
    const halfx8 p0 = pack8_f16(s, 0), p1 = pack8_f16(s, 8);
#pragma unroll
    for (int db = 0; db < kBlocks; ++db) {
      acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[db][0], p0, acc_o[db], 0, 0, 0);
      acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[db][1], p1, acc_o[db], 0, 0, 0);
    }
  };

  // stage t lives in registers raw[t % PF], then in LDS buffer t % 2
  store_stage(ic<0>{}, ic<0>{});
  if (PF < n_stages) load_stage(ic<0>{}, PF);
  __syncthreads();
  for (int t0 = 0; t0 < n_stages; t0 += PF) {
    static_for<0, PF>([&](auto u_c) {
      constexpr int u = decltype(u_c)::value;
      const int t = t0 + u;
      if (t < n_stages) {
        if (t + 1 < n_stages) store_stage(ic<(u + 1) % PF>{}, ic<(u + 1) % 2>{});
        if (t + 1 + PF < n_stages) load_stage(ic<(u + 1) % PF>{}, t + 1 + PF);
        const int j = t * KG + kg;
        if (j < n_tiles && wave_live) compute(j, ic<u % 2>{});
        __syncthreads();
      }
    });
  }

  run_sum = halves_sum(run_sum);
  const int64_t slot = static_cast<int64_t>(split) * p.Hq * p.T + g * M + row0 + c32;
  if constexpr (KG == 1) {
    if (row0 + c32 < M) {
      float* dst = p.part_o + slot * D;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          __builtin_nontemporal_store(floatx4{acc_o[db][4 * r4], acc_o[db][4 * r4 + 1], acc_o[db][4 * r4 + 2], acc_o[db][4 * r4 + 3]},
                                      reinterpret_cast<floatx4*>(dst + 32 * db + 8 * r4 + 4 * hf));
      if (hf == 0) __builtin_nontemporal_store(floatx2{ref, run_sum}, reinterpret_cast<floatx2*>(p.part_ml + slot * 2));
    }
  } else {
    // ---- the key groups' partials of a row block meet in LDS; each group finishes its share of the registers
    constexpr int kRegs = kBlocks * 16;
    float* dump = reinterpret_cast<float*>(lds);
    float* ml = dump + R * KG * kRegs * 64;      // [wave][2][32]
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) dump[(wave * kRegs + db * 16 + r) * 64 + lane] = acc_o[db][r];
    if (hf == 0) {
      ml[wave * 64 + c32] = ref;
      ml[wave * 64 + 32 + c32] = run_sum;
    }
    __syncthreads();
    float weight[KG];
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < KG; ++w) top = fmaxf(top, ml[(w * R + r_block) * 64 + c32]);
#pragma unroll
    for (int w = 0; w < KG; ++w) {
      const float sum = ml[(w * R + r_block) * 64 + 32 + c32];
      weight[w] = sum > 0.f ? fast_exp2(ml[(w * R + r_block) * 64 + c32] - top) : 0.f;     // a group without tiles: nothing
      total = fmaf(sum, weight[w], total);
    }
    if (row0 + c32 < M) {
      float* dst = p.part_o + slot * D;
#pragma unroll
      for (int i = 0; i < kRegs / KG; i += 4) {
        const int first = kg * (kRegs / KG) + i;
        floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KG; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(dump[((w * R + r_block) * kRegs + first + e) * 64 + lane], weight[w], o[e]);
        __builtin_nontemporal_store(o, reinterpret_cast<floatx4*>(dst + 32 * (first >> 4) + 2 * (first & 15) + 4 * hf));
      }
      if (kg == 0 && hf == 0) __builtin_nontemporal_store(floatx2{top, total}, reinterpret_cast<floatx2*>(p.part_ml + slot * 2));
    }
  }
}

template <int D, int R, int KG, int PF, bool SCORES>
hipError_t launch_one(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  auto kernel = prefix_quant_kernel<D, R, KG, PF, SCORES>;
  constexpr int kLdsBytes = lds_bytes<D, R, KG>();
  static_assert(kLdsBytes <= 160 * 1024, "the tiles of a workgroup fit the LDS");
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
  const int groups = (p.M + R * 32 - 1) / (R * 32);
  dim3 grid(p.head_fastest ? p.Hkv : p.S, p.head_fastest ? p.S : p.Hkv, groups);
  return launch_kernel(kernel, grid, dim3(R * KG * 64), kLdsBytes, stream, address_of(p.kp), address_of(p.vp), address_of(p.q), p.kp_sh, p.kp_sl,
                       p.L, p.keys_per_split, p.M, p.G, address_of(s.k), address_of(s.v), s.sh, s.block_log2, p);
}

template <int D, bool SCORES>
hipError_t launch_rows(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  switch (p.rows_per_group) {
    case 32: return launch_one<D, 1, 4, 2, SCORES>(p, s, stream);
    case 64: return launch_one<D, 2, 4, 2, SCORES>(p, s, stream);
    case 128: return launch_one<D, 4, 2, 2, SCORES>(p, s, stream);
    default: return launch_one<D, 8, 1, 4, SCORES>(p, s, stream);
  }
}

}  // namespace

hipError_t launch_prefix_quant(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  if (p.S <= 0) return hipSuccess;
  if (p.d == 128) return p.want_scores ? launch_rows<128, true>(p, s, stream) : launch_rows<128, false>(p, s, stream);
  return p.want_scores ? launch_rows<64, true>(p, s, stream) : launch_rows<64, false>(p, s, stream);
}

}  // namespace specext

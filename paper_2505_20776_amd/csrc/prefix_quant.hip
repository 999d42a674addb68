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
//
// Bound by no single unit: with 256 rows at 32K keys the matrix pipes are busy for 46 % of the time, the vector ALUs (widening,
// exponentials, conversions, addresses) for 53 %, the LDS for 36 %, and under this load the package lowers its clock.  So the steps of
// a tile are laid so that they overlap: behind the barrier the second product of the tile before, from registers, while K comes from
// LDS (128 nodes of 32 heads in 8 groups at 32K keys 71 us per launch, 78 with it in front); then the next tile's logits while V
// comes and the vector ALUs take the exponentials of this one (82 us per attention call, 91 with logits and softmax of one tile behind
// each other).  Now, per launch: 128 nodes 32K 72 us, 0.95 PFLOP/s; 60 nodes 16K 25.5 (cache at 7.08 TB/s 4.8, products at the
// 1.37 PFLOP/s of a large bf16 product 11.8), 2K 11.3; 30 nodes 16K 19.4; 60 nodes of 64-wide heads 8K 12.7.
#include "quant_merge.h"

namespace specext {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((address_space(4))) const float const_float;

constexpr int kTile = 32;      // keys per tile

template <int D>
__host__ __device__ constexpr int tile_bytes() { return kTile * D * 2; }      // K or V of a tile as fp16
constexpr int kPatchStride = 128 * 2 + 8;       // a row of fp16 partials in LDS, padded against bank conflicts
constexpr int kPatchBytes = 32 * kPatchStride;
template <int D, int R, int KG>
constexpr int lds_bytes() {
  const int buffers = 2 * KG * 2 * tile_bytes<D>();
  const int end = KG > 1 ? merge_bytes<D>(R * KG) : D == 128 ? R * kPatchBytes : 0;
  return buffers > end ? buffers : end;
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
  // keys behind the prefix: its last one again, masked below
  auto piece_is_v = [&](int i) { return i * R + r_block >= kPieces / 2; };
  auto piece_row = [&](int i) { return (i * R + r_block) % (kPieces / 2) * kPieceRows + lane / kLanesPerRow; };
  auto piece_there = [&](int i) { return kPieces >= R || i * R + r_block < kPieces; };
  // (offsets within a tile are 32 bits, from a uniform base: no 64-bit products on the vector ALUs)
  const unsigned row_stride = static_cast<unsigned>(kp_sl);
  unsigned in_tile[kPiecesPerWave];
#pragma unroll
  for (int i = 0; i < kPiecesPerWave; ++i) in_tile[i] = piece_row(i) * row_stride + (lane % kLanesPerRow) * 16;
  auto load_piece = [&](int i, int stage) __attribute__((always_inline)) {
    const int key0 = min(key_lo + (stage * KG + kg) * kTile, L - 1);
    const unsigned char* at = (piece_is_v(i) ? vbase : kbase) + key0 * kp_sl;
    unsigned off = in_tile[i];
    if (__builtin_expect(key0 + kTile > L, 0)) off = min(piece_row(i), L - 1 - key0) * row_stride + (lane % kLanesPerRow) * 16;
    return __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(at + off));
  };
  // ---- LDS: per key group two K and two V tiles of 32 rows.  The 16-byte chunks of a row are XOR-swizzled so that the operand
  // reads are free of bank conflicts.
  auto k_swizzle = [](int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); };
  auto v_swizzle = [](int row) { return D == 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); };
  auto store_piece = [&](int i, const uintx4& w, int buf) __attribute__((always_inline)) {
    const int row = piece_row(i);
    const int chunk = 2 * (lane % kLanesPerRow);
    const int swizzle = piece_is_v(i) ? v_swizzle(row) : k_swizzle(row);
    unsigned char* dst = lds + ((kg * 2 + buf) * 2 + (piece_is_v(i) ? 1 : 0)) * kTileBytes + row * kRowBytes;
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) widen4(w[e], h + 2 * e);
    *reinterpret_cast<uintx4*>(dst + ((chunk ^ swizzle) << 4)) = uintx4{h[0], h[1], h[2], h[3]};
    *reinterpret_cast<uintx4*>(dst + (((chunk + 1) ^ swizzle) << 4)) = uintx4{h[4], h[5], h[6], h[7]};
  };
  // Logits are a stage ahead of their softmax, so K is a stage ahead of V: step t brings K of stage t + 1 and V of stage t.
  uintx4 raw[PF][kPiecesPerWave];
  auto load_step = [&](auto slot_c, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPiecesPerWave; ++i)
      if (piece_there(i)) raw[decltype(slot_c)::value][i] = load_piece(i, piece_is_v(i) ? t : t + 1);
  };
  auto store_step = [&](auto slot_c, auto v_buf_c) __attribute__((always_inline)) {
    constexpr int v_buf = decltype(v_buf_c)::value;
#pragma unroll
    for (int i = 0; i < kPiecesPerWave; ++i)
      if (piece_there(i)) store_piece(i, raw[decltype(slot_c)::value][i], piece_is_v(i) ? v_buf : 1 - v_buf);
  };
  uintx4 first_k[kPiecesPerWave];
#pragma unroll
  for (int i = 0; i < kPiecesPerWave; ++i)
    if (piece_there(i) && !piece_is_v(i)) first_k[i] = load_piece(i, 0);
  static_for<0, PF>([&](auto u_c) { load_step(u_c, decltype(u_c)::value); });

  // ---- queries: B operand of S^T (lane = row c32, 8 consecutive d per step), moved to 2^8 at the most
  halfx8 qf[kSteps];
  float c;
  {
    const int m = min(row0 + c32, M - 1);        // padding rows repeat the last real row (never stored)
    const int t = static_cast<int>((static_cast<float>(m) + 0.5f) * (1.0f / static_cast<float>(G)));     // m / G, exact for m < 2^20
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

  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)lds)) + kg * 4 * kTileBytes;
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

  // in registers as they are, instead of an addition per use
#pragma unroll
  for (int ks = 0; ks < kSteps; ++ks) asm volatile("" : "+v"(k_addr[ks]));
#pragma unroll
  for (int db = 0; db < kBlocks; ++db) asm volatile("" : "+v"(v_addr[db]));

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

  // the tile whose softmax comes next
  floatx16 s = {};
  float sk = 0.f, sv = 0.f;      // and its scales
  halfx8 kf[kSteps];
  auto read_k = [&](auto buf_c) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value * 2 * kTileBytes;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
      kf[ks] = __builtin_bit_cast(halfx8, *reinterpret_cast<const lds_uintx4*>(static_cast<uintptr_t>(k_addr[ks] + buf)));
  };
  auto logits = [&](floatx16& x) __attribute__((always_inline)) {
    x = floatx16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[ks], qf[ks], x, 0, 0, 0);
  };
  auto scale_of = [&](const const_float* scale, int j) { return scale[min(key_lo + j * kTile, key_hi - 1) >> block_log2]; };
  // Tile j from its logits in s on, and the logits of tile j + KG into the matrix pipe while the vector ALUs take the exponentials.
  // (Behind the last tile those are of whatever the buffer holds, and nobody reads them: cheaper than a second form of the loop's
  // body, whose registers would spill.)
  halfx8 p0 = {}, p1 = {};       // probabilities of the tile whose second product comes next
  halfx8 vf[2][kBlocks] = {};
  auto read_v = [&](auto buf_c) __attribute__((always_inline)) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) {
        const unsigned at = v_addr[db] + decltype(buf_c)::value * 2 * kTileBytes + 16 * jj * kRowBytes;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)static_cast<uintptr_t>(at));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)static_cast<uintptr_t>(at + 8 * kRowBytes));
        vf[jj][db] = __builtin_bit_cast(halfx8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
  };
  auto second_product = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int db = 0; db < kBlocks; ++db) acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[jj][db], jj ? p1 : p0, acc_o[db], 0, 0, 0);
  };
  auto tile = [&](int j, auto buf_c) __attribute__((always_inline)) {
    const int key0 = key_lo + j * kTile;
    // register r holds key key0 + 8 (r / 4) + 4 hf + r % 4
    if (__builtin_expect(key0 + kTile > key_hi, 0)) {
      const int left = key_hi - key0 - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= left) s[r] = -INFINITY;
    }
    const float ct = c * sk;
    const float lsv = __builtin_amdgcn_logf(sv);
    const float inv_sv = __builtin_amdgcn_rcpf(sv);
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) top = fmaxf(top, fmaxf(s[r], s[r + 1]));
    top = fmaf(top, ct, lsv);                                    // the row's largest, the values' scale included
    if (__builtin_expect(__any(top > ref + kLazyLog2), 0)) {     // some row of this wave outgrew its reference: move every reference up
      settle(acc_o);             // (rare, and the products of the tile before may be just behind)
      const float new_ref = fmaxf(ref, halves_max(top));
      const float alpha = fast_exp2(ref - new_ref);              // 0 on the first tile
      ref = new_ref;
      run_sum *= alpha;
#pragma unroll
      for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc_o[db][r] *= alpha;
    }
    sk = scale_of(k_scale, j + KG), sv = scale_of(v_scale, j + KG);
    read_v(buf_c);
    floatx16 next;
    logits(next);
    const float shift = lsv - ref;
    float part = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(fmaf(s[r], ct, shift));
      part += s[r];
    }
    part *= inv_sv;
    run_sum += part;
    asm volatile("" : "+v"(run_sum));        // here, not behind the next branch
    // every lane stores: the two lanes of a row hold the same pair, and so do padding rows
    if (SCORES) *reinterpret_cast<floatx2*>(score_base + j * score_step + score_off) = floatx2{halves_sum(part), ref};
    p0 = pack8_f16(s, 0), p1 = pack8_f16(s, 8);
    __builtin_amdgcn_sched_group_barrier(0x100, 4 * kBlocks, 0);    // LDS reads
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {                              // a matrix instruction, then its share of the exponentials
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 56 / kSteps, 0);
    }
    // (the products stay here: left to the compiler the last one sinks to the branch in front of the next maxima, see settle())
    asm volatile("" : "+v"(next));
    __builtin_amdgcn_sched_barrier(0);
    s = next;
    __builtin_amdgcn_sched_barrier(0);
  };

#pragma unroll
  for (int i = 0; i < kPiecesPerWave; ++i)
    if (piece_there(i) && !piece_is_v(i)) store_piece(i, first_k[i], 0);
  store_step(ic<0>{}, ic<0>{});
  load_step(ic<0>{}, PF);
  __syncthreads();
  if (kg < n_tiles && wave_live) {
    read_k(ic<0>{});
    logits(s);
    sk = scale_of(k_scale, kg), sv = scale_of(v_scale, kg);
  }
  __syncthreads();
  // Step t of the registers' ring: LDS has V of stage t and K of stage t + 1; what comes next goes where V of t - 1 and K of t were.
  // (Loads behind the last stage repeat the prefix's last row: no branch, and a few bytes from a cache.)
  // Behind a barrier all waves want K from LDS at once, 64 KB for eight of them and 512 cycles; so a tile's second product, its
  // operands in registers, waits for the other side of the barrier and fills the matrix pipe meanwhile, as the next logits do while V
  // comes.
  int t = 0;
  auto step = [&](auto u_c) __attribute__((always_inline)) {
    constexpr int u = decltype(u_c)::value;
    read_k(ic<1 - u % 2>{});
    __builtin_amdgcn_sched_barrier(0);
    second_product();
    store_step(ic<(u + 1) % PF>{}, ic<(u + 1) % 2>{});
    load_step(ic<(u + 1) % PF>{}, t + 1 + PF);
    // the products among the first of the conversions, not as late as their first reader allows (see settle()): 60 nodes at 16K keys
    // 25.4 us per launch, 26.5 with all of them in front of the conversions
#pragma unroll
    for (int i = 0; i < 2 * kBlocks; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
      __builtin_amdgcn_sched_group_barrier(0x002, 1, 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int j = t * KG + kg;
    if (__builtin_expect(wave_live && j < n_tiles, 1)) tile(j, ic<u % 2>{});
    else p0 = p1 = halfx8{};
    __syncthreads();
    ++t;
  };
  // (Whole turns of the ring, then the rest: a loop that is left in its middle has paths that meet, and there the compiler waits for
  // every load in flight.)
  static_assert(PF == 2 || PF == 4, "the rest is written out");
  for (int turns = n_stages / PF; turns > 0; --turns) static_for<0, PF>(step);
  const int rest = n_stages % PF;
  if (rest > 0) {
    step(ic<0>{});
    if constexpr (PF == 4) {
      if (rest > 1) {
        step(ic<1>{});
        if (rest > 2) step(ic<2>{});
      }
    }
  }
  second_product();
  settle(acc_o);

  run_sum = halves_sum(run_sum);
  const int64_t slot = static_cast<int64_t>(split) * p.Hq * p.T + g * M + row0 + c32;
  if constexpr (KG == 1 && D == 128) {
    // ---- fp16 against the row's largest element: the triple (reference, sum, O) is rescaled by the power of two that brings that just
    // below 1, and goes through the wave's own part of LDS, so that whole rows are stored
    float row_max = 0.f;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 2) row_max = fmaxf(row_max, fmaxf(fabsf(acc_o[db][r]), fabsf(acc_o[db][r + 1])));
    row_max = halves_max(row_max);
    const int row_exp = (row_max > 0.f && row_max < INFINITY) ? __builtin_amdgcn_frexp_expf(row_max) : 0;
    const float row_scale = __builtin_amdgcn_ldexpf(1.0f, -row_exp);
    unsigned char* priv = lds + wave * kPatchBytes;
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        uintx2 w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const floatx2 f = {acc_o[db][4 * r4 + 2 * e] * row_scale, acc_o[db][4 * r4 + 2 * e + 1] * row_scale};
          w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, halfx2));
        }
        *reinterpret_cast<uintx2*>(priv + c32 * kPatchStride + (32 * db + 8 * r4 + 4 * hf) * 2) = w;
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    uint16_t* part_h = reinterpret_cast<uint16_t*>(p.part_o) + (slot - c32) * D;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int row = 4 * it + (lane >> 4);
      const uintx2* src = reinterpret_cast<const uintx2*>(priv + row * kPatchStride + 16 * (lane & 15));
      const uintx2 a = src[0], b = src[1];
      if (row0 + row < M) __builtin_nontemporal_store(uintx4{a[0], a[1], b[0], b[1]}, reinterpret_cast<uintx4*>(part_h + row * D + 8 * (lane & 15)));
    }
    if (hf == 0 && row0 + c32 < M)
      __builtin_nontemporal_store(floatx2{ref + static_cast<float>(row_exp), run_sum * row_scale}, reinterpret_cast<floatx2*>(p.part_ml + slot * 2));
  } else if constexpr (KG == 1) {
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
    // ---- the key groups' partials of a row block meet in LDS
    float* dump = reinterpret_cast<float*>(lds);
    dump_wave<D>(dump, R * KG, wave, acc_o, ref, run_sum, lane);
    __syncthreads();
    merge_groups<D, KG>(dump, R * KG, r_block, R, kg, M - row0, p.part_o, p.part_ml, slot - c32, lane);
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
  return p.rows_per_group == 128 ? launch_one<D, 4, 2, 2, SCORES>(p, s, stream) : launch_one<D, 8, 1, 4, SCORES>(p, s, stream);
}

}  // namespace

hipError_t launch_prefix_quant(const AttnParams& p, const QuantScales& s, hipStream_t stream) {
  if (p.S <= 0) return hipSuccess;
  if (p.rows_per_group <= 64) return launch_prefix_quant_few(p, s, stream);
  if (p.d == 128) return p.want_scores ? launch_rows<128, true>(p, s, stream) : launch_rows<128, false>(p, s, stream);
  return p.want_scores ? launch_rows<64, true>(p, s, stream) : launch_rows<64, false>(p, s, stream);
}

}  // namespace specext

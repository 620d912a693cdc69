// Device-side building blocks of the attention kernels: block location, loads into LDS and registers, and the
// transposing reads that feed the second products.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "internal.hpp"

namespace attt {

namespace {
constexpr int DH = 128;     // head dimension
constexpr int BLK = 64;     // query / key rows per block
constexpr int KBLK = kAttnKeyBlock;  // keys per block of a split dK / dV walk
constexpr int PR = DH + 8;  // LDS pitch of a [64][128] tile (bf16): 272 B, conflict-free b128 reads
constexpr float kLog2e = 1.4426950408889634f;

// LDS: two buffers, so that the next block is stored while the current one is read and a step
// needs one barrier. A buffer of the per-query kernels holds the K and V tiles; one of the
// per-key kernels holds the Q and dO tiles, then lse and D of the block's 64 queries.
constexpr int kTileBytes = BLK * PR * 2;
constexpr int kKvBuf = 2 * kTileBytes;
constexpr int kQoBuf = 2 * kTileBytes + 2 * BLK * 4;

__device__ __forceinline__ bf16_t* kv_tile(uint8_t* smem, int buf, int t) {
  return reinterpret_cast<bf16_t*>(smem + buf * kKvBuf + t * kTileBytes);
}
__device__ __forceinline__ bf16_t* qo_tile(uint8_t* smem, int buf, int t) {
  return reinterpret_cast<bf16_t*>(smem + buf * kQoBuf + t * kTileBytes);
}
__device__ __forceinline__ float* qo_stats(uint8_t* smem, int buf) {  // lse [64], then D [64]
  return reinterpret_cast<float*>(smem + buf * kQoBuf + 2 * kTileBytes);
}

__device__ __forceinline__ bf16_t f2bf(float x) { return (bf16_t)(pack_bf16x2(x, 0.0f) & 0xFFFFu); }

// The block a workgroup works on: episode, head, block index. Workgroups start in launch
// order, so the long causal rows go first: the last query blocks for the per-query kernels
// (`late_first`), the first key blocks for the per-key kernel.
__device__ __forceinline__ void attn_locate(const AttnBatch& b, int heads, bool late_first, int& ei, int& head,
                                            int& blk) {
  ei = 0;
  while (ei + 1 < b.count && b.e[ei + 1].wg_begin <= (int)blockIdx.x) ++ei;
  const int local = (int)blockIdx.x - b.e[ei].wg_begin;
  const int nb = b.e[ei].blocks;
  head = local % heads;
  blk = late_first ? nb - 1 - local / heads : local / heads;
}

}  // namespace

// This wave's 16 queries (or keys) as MFMA B operands over the head dimension: lane (l16, q4) holds row
// `row` (its own) at columns 32 s + 8 q4 .. +7 for s = 0..3. Rows at or past nvalid read as zero.
__device__ __forceinline__ void load_row_frags(bf16x8 (&f)[4], const bf16_t* src, int64_t stride, int row,
                                               int nvalid, int q4) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    u32x4 v = u32x4{0u, 0u, 0u, 0u};
    if (row < nvalid) v = *reinterpret_cast<const u32x4*>(src + (int64_t)row * stride + 32 * s + 8 * q4);
    f[s] = __builtin_bit_cast(bf16x8, v);
  }
}

// Rows [0, BLK) of a [rows][DH] block, staged in LDS row-major (pitch PR). Thread tid takes rows
// 4 (tid / 16) .. +3 and columns 8 (tid % 16) .. +7: fetch_block issues its four 16-byte loads
// (rows >= nvalid read as zero), store_block writes them with four 16-byte stores.
// The loads go through one buffer descriptor over the block's valid rows (base and range in
// scalar registers, 32-bit offsets per lane): rows at or past nvalid fall outside its range and
// read as zero. A 64-row block spans less than 2^30 bytes (heads < 2^16, checked on the host).
__device__ __forceinline__ void fetch_block(u32x4 (&v)[4], const bf16_t* src, int64_t stride, int nvalid, int tid) {
  const int r0 = (tid >> 4) * 4, c0 = (tid & 15) * 8;
  const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(src, nvalid > 0 ? (int)(((int64_t)(nvalid - 1) * stride + DH) * 2) : 0);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (uint32_t)(((int64_t)(r0 + i) * stride + c0) * 2), 0, 0));
}

__device__ __forceinline__ void store_block(const u32x4 (&v)[4], bf16_t* dst, int tid) {
  const int r0 = (tid >> 4) * 4, c0 = (tid & 15) * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(dst + (r0 + i) * PR + c0) = v[i];
}

// hi = RN(x), lo = RN(x - hi) of the eight values of an MFMA operand, as bf16x8 pairs.
__device__ __forceinline__ void split_frag(const float (&x)[8], bf16x8& hi, bf16x8& lo) {
  u32x4 h, l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    l[i] = pack_bf16x2(x[2 * i] - bf16_bits_to_f32(h[i] & 0xFFFFu), x[2 * i + 1] - bf16_bits_to_f32(h[i] >> 16));
  }
  hi = __builtin_bit_cast(bf16x8, h);
  lo = __builtin_bit_cast(bf16x8, l);
}

// B operand of the second products over the 32 rows (queries, or keys) of chunk u, from a
// row-major [64][DH] tile (pitch PR) through transposing LDS reads: lane (l16, q4) receives
// column c0 + l16 at rows 32 u + 4 q4 .. +3 and 32 u + 16 + 4 q4 .. +3, the order in which the
// P / dS fragments hold them. ds_read_tr16_b64 hands, within each group of 16 lanes, lane i the
// element i mod 4 of lanes 4e + i/4 (e = 0..3), so lane 4e + c of group q4 addresses row
// 32 u + 4 q4 + e (then 16 rows further) at columns c0 + 4c .. +3.
__device__ __forceinline__ bf16x8 trfrag(const bf16_t* R, int c0, int u, int lane) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s* lds_v4s;
  const int q4 = lane >> 4, e = (lane >> 2) & 3, c = lane & 3;
  const bf16_t* p = R + (32 * u + 4 * q4 + e) * PR + c0 + 4 * c;
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p));
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 16 * PR));
  const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
  return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y});
}

}  // namespace attt

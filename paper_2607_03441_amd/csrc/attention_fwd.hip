// Forward of the adapted attention block over whole prompts (Sec. 3.1's adapted q, k, v, o), and what its
// backward reads of it. Causal attention with grouped key/value heads, packed episodes, head dimension 128:
//   S = scale Q K^T over the keys s <= t of the episode, lse = log sum exp S, O = exp(S - lse) V,
//   D = rowsum(dO * O) for the backward.
// One pass over the keys: the running maximum and sum of the softmax and O stay in registers.
#include "attention_core.hpp"
#include "lds_limit.hpp"

namespace attt {

// The bits 15 and 31 of the halves of x that hold an infinity or a NaN (exponent bits all set).
__device__ __forceinline__ uint32_t nonfinite_halves(uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }

// Whether a [64][128] tile holds one: this lane's sixteen 16-byte pieces of it.
__device__ __forceinline__ bool any_nonfinite(const bf16_t* R, int lane) {
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(R + (4 * i + (lane >> 4)) * PR + 8 * (lane & 15));
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= nonfinite_halves(x[e]);
  }
  return odd != 0;
}

__device__ __forceinline__ bf16x8 without_nonfinite(bf16x8 f) {
  u32x4 x = __builtin_bit_cast(u32x4, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] &= ~((nonfinite_halves(x[e]) >> 15) * 0xFFFFu);
  return __builtin_bit_cast(bf16x8, x);
}

// O and lse of one (query head, 64 QT-query block). Wave w owns queries 16 QT w .. + 16 QT - 1 as QT tiles of
// 16, their Q fragments in registers as the B operand of S^T = K Q^T, so that each lane holds 16 scores of
// its own query of a tile. exp(S - m), rounded to bf16 once (it is a weight in [0, 2^8]; the
// rounding's 2^-9 is that of O itself), is then directly the B operand of O^T = V^T P^T: the contraction
// runs over the keys in the order the lane holds them, and V^T comes from the row-major V tile through
// transposing reads in that order. A lane's O values are all of its own query, so the factor by which an
// older maximum is replaced is one register per tile. It is applied only where a maximum has grown by more than
// 2^8: until then the weights stay below 2^8, which costs no precision in float32 or bf16.
template <int QT>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnArgs a, AttnBatch b) {
  constexpr int QBLK = 64 * QT;
  int ei, h, qb;
  attn_locate(b, a.heads, true, ei, h, qb);
  const AttnEp E = b.e[ei];
  const int kh = h / (a.heads / a.kv_heads);
  const int q0 = qb * QBLK, nq = min(QBLK, E.L - q0);
  extern __shared__ __align__(16) uint8_t smem[];  // two buffers of [K tile][V tile], [64][PR] each
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, q4 = lane >> 4;
  const int64_t qs = (int64_t)a.heads * DH, ks = (int64_t)a.kv_heads * DH;
  bf16x8 qf[QT][4];
#pragma unroll
  for (int c = 0; c < QT; ++c)
    load_row_frags(qf[c], a.q + ((int64_t)(E.row0 + q0) * a.heads + h) * DH, qs, 16 * QT * w + 16 * c + l16, nq, q4);
  const float sl = a.scale * kLog2e;
  float m[QT], l[QT];  // base 2; m the same in the query's four lanes, l this lane's share
  f32x4 o[QT][8];
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    m[c] = -INFINITY, l[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[c][j] = f32x4{0, 0, 0, 0};
  }
  u32x4 fk[4], fv[4];
  auto fetch = [&](int kb) {
    const int k0 = kb * BLK, nk = min(BLK, E.L - k0);
    fetch_block(fk, a.k + ((int64_t)(E.row0 + k0) * a.kv_heads + kh) * DH, ks, nk, tid);
    fetch_block(fv, a.v + ((int64_t)(E.row0 + k0) * a.kv_heads + kh) * DH, ks, nk, tid);
  };
  const int kb_last = (q0 + nq - 1) / BLK;  // the key block of the block's last query
  const int wq0 = q0 + 16 * QT * w;         // this wave's first query
  fetch(0);
  store_block(fk, kv_tile(smem, 0, 0), tid);
  store_block(fv, kv_tile(smem, 0, 1), tid);
  for (int kb = 0; kb <= kb_last; ++kb) {
    const int k0 = kb * BLK;
    // This block's tiles are stored, and every wave is done with the other buffer.
    __syncthreads();
    if (kb < kb_last) fetch(kb + 1);  // the next key block loads while this one computes
    // A wave whose queries all precede the block has nothing to add.
    if (k0 <= wq0 + 16 * QT - 1) {
      const bf16_t* Ks = kv_tile(smem, kb & 1, 0);
      const bf16_t* Vs = kv_tile(smem, kb & 1, 1);
      f32x4 st[QT][4];  // S^T[16 tt + 4 q4 + r][query]
#pragma unroll
      for (int c = 0; c < QT; ++c)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) st[c][tt] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
          const bf16x8 ak = __builtin_bit_cast(
              bf16x8, *reinterpret_cast<const u32x4*>(Ks + (16 * tt + l16) * PR + 32 * s4 + 8 * q4));
#pragma unroll
          for (int c = 0; c < QT; ++c) st[c][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ak, qf[c][s4], st[c][tt], 0, 0, 0);
        }
      bf16x8 p[QT][2];  // weights of keys 32 u + 4 q4 .. +3 and 32 u + 16 + 4 q4 .. +3
      // A key block that ends at or before the wave's first query is whole and entirely allowed: no mask there.
      auto softmax = [&](auto masked) {
#pragma unroll
        for (int c = 0; c < QT; ++c) {
          float mx = -INFINITY;
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float v = st[c][tt][r] * sl;
              // keys past the episode come after every query of it
              if constexpr (decltype(masked)::value) v = k0 + 16 * tt + 4 * q4 + r <= wq0 + 16 * c + l16 ? v : -INFINITY;
              st[c][tt][r] = v;
              mx = fmaxf(mx, v);
            }
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          if (__any(mx > m[c] + 8.0f)) {
            const float mn = mx > m[c] + 8.0f ? mx : m[c];  // per row: no other row of the tile changes it
            const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[c] - mn);
            m[c] = mn;
            l[c] *= alpha;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[c][j] *= alpha;
          }
          const float ms = m[c] == -INFINITY ? 0.0f : m[c];  // no key yet, or only scores of -inf: their weights are 0
          float sum = 0.0f;
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              st[c][tt][r] = __builtin_amdgcn_exp2f(st[c][tt][r] - ms);
              sum += st[c][tt][r];
            }
          l[c] += sum;
#pragma unroll
          for (int u = 0; u < 2; ++u)
            p[c][u] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(st[c][2 * u][0], st[c][2 * u][1]),
                                                       pack_bf16x2(st[c][2 * u][2], st[c][2 * u][3]),
                                                       pack_bf16x2(st[c][2 * u + 1][0], st[c][2 * u + 1][1]),
                                                       pack_bf16x2(st[c][2 * u + 1][2], st[c][2 * u + 1][3])});
        }
      };
      const bool whole = k0 + BLK - 1 <= wq0;
      if (whole)
        softmax(std::false_type{});
      else
        softmax(std::true_type{});
      auto product = [&](auto clean) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            bf16x8 av = trfrag(Vs, 16 * j, u, lane);
            if constexpr (decltype(clean)::value) av = without_nonfinite(av);
#pragma unroll
            for (int c = 0; c < QT; ++c) o[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, p[c][u], o[c][j], 0, 0, 0);
          }
      };
      // Where some queries do not see all keys, a weight of 0 does not hide an infinity or a NaN in V from the
      // product. Such entries are left out of it and added to the queries that see them.
      if (!whole && __any(any_nonfinite(Vs, lane))) {
        product(std::true_type{});
#pragma unroll 1
        for (int s = 0; s < BLK; ++s)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint2 x = *reinterpret_cast<const uint2*>(Vs + s * PR + 16 * j + 4 * q4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = bf16_bits_to_f32((r < 2 ? x.x : x.y) >> (r & 1 ? 16 : 0) & 0xFFFFu);
              if (__builtin_isfinite(v)) continue;
#pragma unroll
              for (int c = 0; c < QT; ++c)
                if (k0 + s <= wq0 + 16 * c + l16) o[c][j][r] += v;
            }
          }
      } else {
        product(std::false_type{});
      }
    }
    if (kb < kb_last) {
      store_block(fk, kv_tile(smem, (kb + 1) & 1, 0), tid);
      store_block(fv, kv_tile(smem, (kb + 1) & 1, 1), tid);
    }
  }
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    const int qry = 16 * QT * w + 16 * c + l16;
    float lc = l[c];
    lc += __shfl_xor(lc, 16, 64);
    lc += __shfl_xor(lc, 32, 64);
    if (qry < nq) {
      if (q4 == 0) a.lse[(int64_t)h * a.N + E.row0 + q0 + qry] = m[c] / kLog2e + logf(lc);
      const float inv = 1.0f / lc;
      bf16_t* orow = a.o + ((int64_t)(E.row0 + q0 + qry) * a.heads + h) * DH;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint2*>(orow + 16 * j + 4 * q4) =
            make_uint2(pack_bf16x2(o[c][j][0] * inv, o[c][j][1] * inv), pack_bf16x2(o[c][j][2] * inv, o[c][j][3] * inv));
    }
  }
}

// D = rowsum(dO * O) of every (row, query head), 16 lanes each: dsum [heads][N].
__global__ __launch_bounds__(256) void attn_dsum_kernel(AttnArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);  // row-major (row, head)
  const int c0 = (threadIdx.x & 15) * 8;
  if (i >= (int64_t)a.N * a.heads) return;
  const u32x4 x = *reinterpret_cast<const u32x4*>(a.o + i * DH + c0), y = *reinterpret_cast<const u32x4*>(a.dout + i * DH + c0);
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s = fmaf(bf16_bits_to_f32(x[e] & 0xFFFFu), bf16_bits_to_f32(y[e] & 0xFFFFu), s);
    s = fmaf(bf16_bits_to_f32(x[e] >> 16), bf16_bits_to_f32(y[e] >> 16), s);
  }
  s = group_sum<16>(s);
  if ((threadIdx.x & 15) == 0) a.dsum[(i % a.heads) * a.N + i / a.heads] = s;
}

template <int QT>
static hipError_t launch_fwd(LdsLimit& limit, const AttnArgs& a, AttnBatch b, hipStream_t s) {
  constexpr size_t lds = 2 * (size_t)kKvBuf;
  if (hipError_t e = limit.raise((const void*)attn_fwd_kernel<QT>, lds)) return e;
  int n = 0;
  for (int i = 0; i < b.count; ++i) {
    b.e[i].blocks = (b.e[i].L + 64 * QT - 1) / (64 * QT);
    b.e[i].wg_begin = n;
    n += b.e[i].blocks * a.heads;
  }
  if (n <= 0) return hipSuccess;
  KernelTimer t(K_ATTN_PROMPT, s);
  hipLaunchKernelGGL(attn_fwd_kernel<QT>, dim3(n), dim3(256), lds, s, a, b);
  return hipGetLastError();
}

hipError_t launch_attn_fwd(const AttnArgs& a, const AttnBatch& b, hipStream_t s) {
  static LdsLimit limits[2];
  int n1 = 0, n2 = 0;
  for (int i = 0; i < b.count; ++i) n1 += (b.e[i].L + 63) / 64, n2 += (b.e[i].L + 127) / 128;
  const bool wide = (int64_t)n2 * a.heads > 480 && 8 * (int64_t)n1 > 9 * (int64_t)n2;
  return wide ? launch_fwd<2>(limits[1], a, b, s) : launch_fwd<1>(limits[0], a, b, s);
}

hipError_t launch_attn_dsum(const AttnArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.N * a.heads;
  KernelTimer t(K_ATTN_DSUM, s);
  hipLaunchKernelGGL(attn_dsum_kernel, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace attt

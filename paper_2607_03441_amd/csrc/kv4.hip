// Serving: a key/value cache in 4 bits and the attention over it, for concurrent episodes that decode over
// long histories (Appendix A).
//
// The cache is paged: per page of 128 tokens and key/value head one record of kKv4Record bytes, laid out for the
// reads of the attention kernel, whose lane (l16, q4) of a wave takes in every load 16 bytes that it
// multiplies itself:
//   keys    e2m1 codes [128 tokens][64 bytes], two a byte along the head dimension. Every 32 elements share a power of two
//           2^(b - 127); the bytes b lie at [block of 32][token % 16][token / 16], so that lane (l16, q4)
//           gets those of its 8 tokens 16 i + l16 and its block q4 with one 8-byte load.
//   values  e2m1 codes [128 elements][64 bytes], two a byte along the tokens: position 32 a + 4 b + c of a row
//           is token 16 b + 4 a + c. That is the order in which the score products leave a lane's weights, so
//           they enter the second product without a move between lanes.
//           One scale per token (bf16 with 6 significant bits), in the same order: it goes into the
//           weight, because the contraction runs over the tokens.
// Codes times scales have at most 8 significant bits, so the bf16 operands of the products are exact.
#include <type_traits>

#include "common.hpp"
#include "internal.hpp"
#include "lds_limit.hpp"

namespace attt {

namespace {
constexpr int DH = 128;
constexpr int kPage = kKv4Page, kRec = kKv4Record;
constexpr int kOffV = kPage * DH / 2, kOffKs = 2 * kOffV, kOffVs = kOffKs + kPage * 4;
static_assert(kOffVs + kPage * 2 == kRec, "the record's parts");
constexpr size_t kChunkBuf = kOffKs + 1024;  // a page in LDS
constexpr float kLog2e = 1.4426950408889634f;

// Sequence of workgroup `bid`: the last whose wg_begin is at most bid. Where all have the same rows (decoding), none of
// the batch's entries needs to be read for it.
__device__ __forceinline__ Kv4Seq find_seq(const Kv4Batch& b, int bid) {
  if (b.same) {
    const int e = bid / b.wgs;
    return {b.s[0].row0 + (int64_t)e * b.same, b.same, b.s[0].seq + e, e * b.wgs, b.s[0].blk0 + e * b.blocks};
  }
  const int lane = threadIdx.x & 63;
  return b.s[__builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < b.count && b.s[lane < b.count ? lane : 0].wg_begin <= bid)) - 1)];
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// eight e2m1 codes times a scale as bf16 (exact)
__device__ __forceinline__ bf16x8 widen(uint32_t x, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3)};
  return bf16x8{y[0][0], y[0][1], y[1][0], y[1][1], y[2][0], y[2][1], y[3][0], y[3][1]};
}
}  // namespace

// The new rows of one (sequence, key/value head) that fall into one page and there onto the tokens 16 i + 4 q + r of one q:
// those 32 make up one 16-byte piece of every value row, so no two workgroups write into one piece. Sixteen lanes take a
// token, eight elements each, two tokens after the other with both loads on their way: the maxima of its key blocks
// (4 lanes) and of its value row (16 lanes) meet in shuffles. Key codes go to the page at once; value codes are
// turned through LDS, and each piece is written by one thread, which keeps the codes of the tokens that were there.
// Bound by memory: 16 x 512 rows of 8 heads, 76 MB with what they stand for, in 18 us, 4.2 TB/s. (A workgroup per page, 16
// tokens at a time, took 44 us.) One row of each of 16 sequences takes 5 us, the latency of length, page id and page.
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Args a, Kv4Batch b) {
  const Kv4Seq S = find_seq(b, blockIdx.x);
  const int local = (int)blockIdx.x - S.wg_begin;
  // the four pieces of a page and head eight workgroups apart, on one XCD, whose L2 puts their writes into whole lines
  const int q = local >> 3 & 3, unit = (local >> 5) * 8 + (local & 7), kh = unit % a.kv_heads, nth = unit / a.kv_heads;
  const int lane16 = threadIdx.x & 15;
  u32x4 xk[2], xv[2];
  if (S.n == 1) {  // the one row is known before the length is
    const int64_t at = (S.row0 * a.kv_heads + kh) * DH + lane16 * 8;
    xk[0] = xk[1] = *reinterpret_cast<const u32x4*>(a.k + at);
    xv[0] = xv[1] = *reinterpret_cast<const u32x4*>(a.v + at);
  }
  const int64_t len = a.lengths[S.seq];
  const int64_t first = len - S.n;  // position of the sequence's first new row; rows before 0 are not stored
  const int64_t page = (first > 0 ? first : 0) / kPage + nth;
  const bool bad_len = len > a.width * kPage;
  __shared__ __align__(16) uint8_t codes[DH][32 + 16];  // value codes by (element, place in the piece)
  const int tid = threadIdx.x;
  const bool held = a.k_held != nullptr;
  if (nth >= (S.n + kPage - 2) / kPage + 1) return;
  if (nth == 0 && q == 0 && held) {
    // what the sequence has no place for: rows before its start hold nothing, those of a bad length NaN
    const int none = bad_len ? S.n : (int)min((int64_t)S.n, max((int64_t)0, -first));
    const uint32_t fill = bad_len ? 0x7FC07FC0u : 0u;
    for (int i = tid >> 4; i < none; i += 16) {
      const int64_t at = ((S.row0 + i) * a.kv_heads + kh) * DH + lane16 * 8;
      *reinterpret_cast<u32x4*>(a.k_held + at) = u32x4{fill, fill, fill, fill};
      *reinterpret_cast<u32x4*>(a.v_held + at) = u32x4{fill, fill, fill, fill};
    }
  }
  // tokens [t0, t1) of the page are new
  const int t0 = (int)max((int64_t)0, max((int64_t)0, first) - page * kPage), t1 = (int)min((int64_t)kPage, len - page * kPage);
  // a run of tokens touches pieces t0 / 4, t0 / 4 + 1, ... in turn
  if (bad_len || t0 >= t1 || ((q - (t0 >> 2)) & 3) > ((t1 - 1) >> 2) - (t0 >> 2)) return;
  // this thread's tokens: places 16 u + tid / 16 of the piece, 4 i + r of token 16 i + 4 q + r
  int t[2];
  bool on[2];
  int64_t at[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int place = 16 * u + (tid >> 4);
    t[u] = 16 * (place >> 2) + 4 * q + (place & 3);
    on[u] = t[u] >= t0 && t[u] < t1;
    at[u] = ((S.row0 + (on[u] ? page * kPage + t[u] - first : 0)) * a.kv_heads + kh) * DH + lane16 * 8;
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (S.n == 1) break;
    xk[u] = *reinterpret_cast<const u32x4*>(a.k + at[u]);
    xv[u] = *reinterpret_cast<const u32x4*>(a.v + at[u]);
  }
  const int id = a.table[S.seq * a.width + page];
  const bool stored = id >= 0 && id < a.pages;
  uint8_t* rec = a.cache + ((int64_t)(stored ? id : 0) * a.kv_heads + kh) * kRec;
  u32x4* piece = reinterpret_cast<u32x4*>(rec + kOffV + (tid & (DH - 1)) * 64 + q * 16);
  u32x4 was = u32x4{0, 0, 0, 0};
  if (stored && tid < DH && t1 - t0 < kPage) was = *piece;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (!__any(on[u])) continue;
    uint32_t mk = 0, mv = 0;  // the largest magnitude, as bits: NaN above infinity above the rest
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mk = max(mk, max(xk[u][e] << 16 & 0x7FFF0000u, xk[u][e] & 0x7FFF0000u));
      mv = max(mv, max(xv[u][e] << 16 & 0x7FFF0000u, xv[u][e] & 0x7FFF0000u));
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      if (o < 4) mk = max(mk, (uint32_t)__shfl_xor((int)mk, o, 64));
      mv = max(mv, (uint32_t)__shfl_xor((int)mv, o, 64));
    }
    // keys: the power of two that leaves the largest of 32 below 7 (6, the largest code, is nearer to it than 8
    // times half of it): the exponent, less 2, rounded up from 1.75; at least 2^-100, and 6 times it is finite.
    const bool nan_k = mk >= 0x7F800000u, nan_v = mv >= 0x7F800000u;
    const uint32_t ek = nan_k ? 255u : min(252, max(27, (int)((mk + 0x200000u) >> 23) - 2));
    const float sk = __uint_as_float((nan_k ? 127u : ek) << 23);
    // values: a sixth of the largest, rounded up to 6 significant bits, so that the largest is 6 at most
    // (bounded like the keys')
    const float sixth = __fdiv_rn(nan_v ? 1.0f : __uint_as_float(mv), 6.0f);
    const float sv = fminf(fmaxf(__uint_as_float((__float_as_uint(sixth) + 0x3FFFFu) & ~0x3FFFFu), 0x1p-100f), 0x1.5p125f);
    // The matrix core's own conversions round to nearest, ties to the even code, and stop at 6. A value over its scale
    // is first rounded to float32, with one correction of the product with the reciprocal: a quotient that lies
    // on the border of two codes is exact then, and any other is at least 2^-9 of itself away from one.
    const float rv = __fdiv_rn(1.0f, sv);
    uint32_t wk = 0, wv = 0;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    auto pair = [&](uint32_t x, auto sel) {
      const float lo = bf16_bits_to_f32(x & 0xFFFFu), hi = __uint_as_float(x & 0xFFFF0000u);
      auto over = [&](float x) {
        const float y = x * rv;
        return copysignf(fmaf(fmaf(-y, sv, x), rv, y), x);  // a zero keeps its sign
      };
      wv = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(wv, over(lo), over(hi), 1.0f, decltype(sel)::value);
    };
    auto pair_k = [&](uint32_t x, auto sel) {
      wk = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(wk, bf16_bits_to_f32(x & 0xFFFFu), __uint_as_float(x & 0xFFFF0000u), sk,
                                                    decltype(sel)::value);
    };
    pair_k(xk[u][0], std::integral_constant<int, 0>{}), pair(xv[u][0], std::integral_constant<int, 0>{});
    pair_k(xk[u][1], std::integral_constant<int, 1>{}), pair(xv[u][1], std::integral_constant<int, 1>{});
    pair_k(xk[u][2], std::integral_constant<int, 2>{}), pair(xv[u][2], std::integral_constant<int, 2>{});
    pair_k(xk[u][3], std::integral_constant<int, 3>{}), pair(xv[u][3], std::integral_constant<int, 3>{});
    if (nan_k) wk = 0;
    if (nan_v) wv = 0;
    const int place = 16 * u + (tid >> 4);
    if (on[u] && stored) {
      *reinterpret_cast<uint32_t*>(rec + t[u] * 64 + lane16 * 4) = wk;
      if ((lane16 & 3) == 0) rec[kOffKs + (lane16 >> 2) * 128 + (t[u] & 15) * 8 + (t[u] >> 4)] = (uint8_t)ek;
      if (lane16 == 0)
        *reinterpret_cast<uint16_t*>(rec + kOffVs + 2 * (32 * q + place)) = nan_v ? 0x7FC0 : (uint16_t)(__float_as_uint(sv) >> 16);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) codes[lane16 * 8 + e][place] = (uint8_t)(wv >> (4 * e) & 15u);
    if (on[u] && held) {
      u32x4 hk = __builtin_bit_cast(u32x4, widen(wk, sk)), hv;
      auto value = [&](int e, auto sel) {
        const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wv, 1.0f, decltype(sel)::value);
        hv[e] = pack_bf16x2(y[0] * sv, y[1] * sv);
      };
      value(0, std::integral_constant<int, 0>{}), value(1, std::integral_constant<int, 1>{});
      value(2, std::integral_constant<int, 2>{}), value(3, std::integral_constant<int, 3>{});
      const u32x4 nan = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
      *reinterpret_cast<u32x4*>(a.k_held + at[u]) = nan_k || !stored ? nan : hk;
      *reinterpret_cast<u32x4*>(a.v_held + at[u]) = nan_v || !stored ? nan : hv;
    }
  }
  __syncthreads();
  if (!stored || tid >= DH) return;
  u32x4 w, keep = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int half = 0; half < 2; ++half) {  // 16 codes, a byte each, become 8 bytes
    const u32x4 x = *reinterpret_cast<const u32x4*>(&codes[tid][16 * half]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t lo = x[2 * e] | x[2 * e] >> 4, hi = x[2 * e + 1] | x[2 * e + 1] >> 4;  // pairs in bytes 0 and 2
      w[2 * half + e] = (lo & 0xFFu) | (lo >> 8 & 0xFF00u) | (hi & 0xFFu) << 16 | (hi << 8 & 0xFF000000u);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int tok = 16 * i + 4 * q + r;
      if (tok < t0 || tok >= t1) keep[i >> 1] |= 0xFu << (16 * (i & 1) + 4 * r);
    }
  *piece = (w & ~keep) | (was & keep);
}

namespace {
// What a workgroup of the attention works on: rows rb R .. of a head's group (row i g + j: token i, query head j),
// pages [p0, p1) of the sequence.
struct Kv4Work {
  Kv4Seq S;
  int kh, split, rb, g, p0, p1;
  int64_t first;  // position of the sequence's first new row
  bool bad;       // a length beyond the bound: the rows are NaN
  // whether there is nothing to write either
  __device__ __forceinline__ bool locate(const Kv4Args& a, const Kv4Batch& b) {
    S = find_seq(b, blockIdx.x);
    const int local = (int)blockIdx.x - S.wg_begin;
    kh = local % a.kv_heads;
    const int sb = local / a.kv_heads;
    g = a.heads / a.kv_heads;
    // a split's row blocks side by side: they read the same pages, through one XCD's L2 where kv_heads is a multiple of 8
    const int blocks = (S.n * g + a.block_rows - 1) / a.block_rows;
    rb = sb % blocks;
    split = sb / blocks;
    int64_t len = a.lengths[S.seq];
    bad = len > a.max_length;
    if (len < 0 || bad) len = 0;
    p0 = split * a.chunk;
    p1 = min((int)((len + kPage - 1) / kPage), p0 + a.chunk);
    first = len - S.n;
    return split > 0 && p0 >= p1;  // not among those that are joined
  }
};

// One row tile's query rows as B operands, in the order in which a lane holds its keys' codes; the last position that
// the lane's row sees (-1: none). Rows past the sequence's are zero.
__device__ __forceinline__ int load_rows(bf16x8 (&qf)[4], const Kv4Args& a, const Kv4Work& k, int row, int q4) {
  const int i = row / k.g, j = row % k.g;
  const bool on = row < k.S.n * k.g;
  const bf16_t* src = a.q + ((k.S.row0 + (on ? i : 0)) * a.heads + k.kh * k.g + (on ? j : 0)) * DH + 32 * q4;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(src + 8 * s);
    qf[s] = __builtin_bit_cast(bf16x8, on ? x : u32x4{0, 0, 0, 0});
  }
  return on ? (int)max((int64_t)-1, k.first + i) : -1;
}

// The online softmax of PT tiles of 16 tokens, the lane's being t0 + 16 i + r, for one row tile: scores in, weights
// times the value scales (pairs in `scale`, bf16 bits, in the order of the value rows) out, rounded to bf16 once.
// An older maximum is replaced only where it is passed by more than 2^8.
template <int PT, bool MASKED>
__device__ __forceinline__ void weigh(f32x4 (&st)[PT], bf16x8 (&pw)[PT / 2], const u32x4* scale, float sl, int t0, int lim, float& m,
                                      float& l, f32x4 (&o)[8]) {
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < PT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (MASKED) st[i][r] = t0 + 16 * i + r <= lim ? st[i][r] : -INFINITY;
      mx = fmaxf(mx, st[i][r]);
    }
  mx = rows_max(mx) * sl;
  if (__any(mx > m + 8.0f)) {
    const float mn = mx > m + 8.0f ? mx : m;  // per row: no other row of the tile changes it
    const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= alpha;
  }
  const float ms = m == -INFINITY ? 0.0f : m;
  float sum = 0.0f;
  u32x4 pk[PT / 2];
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    float x[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(fmaf(st[i][r], sl, -ms));
      sum += e;
      const uint32_t pair = scale[i >> 1][(i & 1) * 2 + (r >> 1)];
      x[r] = e * __uint_as_float(r & 1 ? pair & 0xFFFF0000u : pair << 16);
      // places that no token was written to hold any bits
      if constexpr (MASKED) x[r] = t0 + 16 * i + r <= lim ? x[r] : 0.0f;
    }
    pk[i >> 1][(i & 1) * 2] = pack_bf16x2(x[0], x[1]);
    pk[i >> 1][(i & 1) * 2 + 1] = pack_bf16x2(x[2], x[3]);
  }
  l += sum;
#pragma unroll
  for (int u = 0; u < PT / 2; ++u) pw[u] = __builtin_bit_cast(bf16x8, pk[u]);
}

// Writes a row tile's result: o and lse, or with several splits O's sums, the maximum and the sum of weights.
__device__ __forceinline__ void write_rows(const Kv4Args& a, const Kv4Work& k, int in_block, float m, float l, const f32x4 (&o)[8], int q4) {
  const int row = k.rb * a.block_rows + in_block, i = row / k.g, j0 = row % k.g;
  if (row >= k.S.n * k.g) return;
  if (a.splits > 1) {
    const int64_t at = (((int64_t)(k.S.blk0 + k.rb) * a.kv_heads + k.kh) * a.splits + k.split) * a.block_rows + in_block;
#pragma unroll
    for (int j = 0; j < 8; ++j) *reinterpret_cast<f32x4*>(a.part + at * DH + 16 * j + 4 * q4) = o[j];
    if (q4 == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  const int h = k.kh * k.g + j0;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // a row that sees nothing: 0, lse -inf
  if (q4 == 0) a.lse[(int64_t)h * a.N + k.S.row0 + i] = l == 0.0f ? -INFINITY : m / kLog2e + logf(l);
  bf16_t* dst = a.o + ((k.S.row0 + i) * a.heads + h) * DH + 4 * q4;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<uint2*>(dst + 16 * j) = make_uint2(pack_bf16x2(o[j][0] * inv, o[j][1] * inv), pack_bf16x2(o[j][2] * inv, o[j][3] * inv));
}
}  // namespace

// Attention of at most 16 query rows per workgroup (decoding steps): the four waves take whole pages in turn. The
// rows are the columns of S^T = K Q^T, so each lane holds 32 scores of its own row per page; the softmax is a reduction over
// the lane's registers and its three partner lanes. Weight times value scale is the B operand of O^T = V^T P^T. A
// page's keys are asked for while the one before is multiplied with its values, and its values while
// its keys are. At the end the waves' sums are joined in a fixed order through LDS.
// Bound by the reads: one row of 8 episodes of 8192 to 131072 tokens (32 heads over 8) 632 MB in 117 us, 5.4 TB/s. At up to
// 4000 tokens of 16 episodes 38 MB in 12.5 us: the latency of length, page id, page and product one after the other (page
// ids and rows asked for before the length is known: the same).
__global__ __launch_bounds__(256, 2) void kv4_decode_kernel(Kv4Args a, Kv4Batch b) {
  Kv4Work k;
  if (k.locate(a, b)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, q4 = lane >> 4;
  bf16x8 qf[4];
  const int lim = load_rows(qf, a, k, k.rb * 16 + l16, q4);
  const int64_t all_see = k.first + (k.rb * 16) / k.g;  // every row of the block sees the positions up to here
  const float sl = a.scale * kLog2e;
  float m = -INFINITY, l = 0.0f;
  f32x4 o[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = f32x4{0, 0, 0, 0};
  u32x4 kr[8], vr[8], vs[4];
  uint2 ks;
  const int32_t* table = a.table + (int64_t)k.S.seq * a.width;
  bool bad = k.bad;
  auto record = [&](int p) -> const uint8_t* {
    int id = table[p];
    if (id < 0 || id >= a.pages) bad = true, id = 0;
    return a.cache + ((int64_t)id * a.kv_heads + k.kh) * kRec;
  };
  auto load_k = [&](const uint8_t* rec) {
#pragma unroll
    for (int i = 0; i < 8; ++i) kr[i] = *reinterpret_cast<const u32x4*>(rec + (16 * i + l16) * 64 + 16 * q4);
    ks = *reinterpret_cast<const uint2*>(rec + kOffKs + 128 * q4 + 8 * l16);
  };
  auto load_v = [&](const uint8_t* rec) {
#pragma unroll
    for (int j = 0; j < 8; ++j) vr[j] = *reinterpret_cast<const u32x4*>(rec + kOffV + (16 * j + l16) * 64 + 16 * q4);
#pragma unroll
    for (int i = 0; i < 4; ++i) vs[i] = *reinterpret_cast<const u32x4*>(rec + kOffVs + 64 * q4 + 16 * i);
  };
  int p = k.p0 + w;
  const uint8_t* rec = nullptr;
  if (p < k.p1) {
    rec = record(p);
    load_k(rec);
    load_v(rec);
  }
  auto page = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const bool more = p + 4 < k.p1;
    const uint8_t* next = more ? record(p + 4) : rec;
    f32x4 st[8];  // S^T[16 i + 4 q4 + r][row]
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      st[i] = f32x4{0, 0, 0, 0};
      const float sc = __uint_as_float(((i < 4 ? ks.x : ks.y) >> (8 * (i & 3)) & 255u) << 23);
#pragma unroll
      for (int s = 0; s < 4; ++s) st[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(kr[i][s], sc), qf[s], st[i], 0, 0, 0);
    }
    if (more) load_k(next);
    bf16x8 pw[4];
    weigh<8, MASKED>(st, pw, vs, sl, p * kPage + 4 * q4, lim, m, l, o);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(vr[j][u], 1.0f), pw[u], o[j], 0, 0, 0);
    if (more) load_v(next);
    rec = next;
  };
  // pages that every row sees first: masks behind a branch in one loop made the compiler copy O in every step
  for (; p < k.p1 && (int64_t)p * kPage + kPage - 1 <= all_see; p += 4) page(std::false_type{});
  for (; p < k.p1; p += 4) page(std::true_type{});
  // the four waves' maxima, sums and O: waves 2 and 3 hand over to 0 and 1, then 1 to 0
  __shared__ f32x4 ex[2][8][64];
  __shared__ float2 ml[2][64];
  l = rows_sum(l);
  if (bad) l = __uint_as_float(0x7FC00000u);
#pragma unroll
  for (int step = 2; step > 0; step >>= 1) {
    __syncthreads();
    if (w >= step && w < 2 * step) {
      ml[w - step][lane] = make_float2(m, l);
#pragma unroll
      for (int j = 0; j < 8; ++j) ex[w - step][j][lane] = o[j];
    }
    __syncthreads();
    if (w < step) {
      const float2 other = ml[w][lane];
      const float mn = fmaxf(m, other.x), ms = mn == -INFINITY ? 0.0f : mn;
      const float fa = __builtin_amdgcn_exp2f(m - ms), fb = __builtin_amdgcn_exp2f(other.x - ms);
      m = mn;
      l = l * fa + other.y * fb;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = o[j] * fa + ex[w][j][lane] * fb;
    }
  }
  if (w == 0) write_rows(a, k, l16, m, l, o, q4);
}

// Attention of 128 query rows per workgroup (prompts in chunks): every wave owns two tiles of 16 rows and goes over all
// pages of the split, which lie in LDS as they are in the cache, the next one on its way. Nothing is joined between the waves.
// Bound by issue: every wave widens all codes and takes its exponentials, and two waves share a SIMD. 64 rows of 4
// sequences of 512 to 8200 tokens (32 heads over 8) 46 us with the join. On the way there: pages in each wave's registers
// instead of LDS 80, here 56; two sets of four waves on alternate pages 61; one row tile a wave 57; a split's row blocks side
// by side 50; no copies of O (see the loops) 47; V asked for before the exponentials 46. Four row tiles a wave spill.
__global__ __launch_bounds__(256, 2) void kv4_chunk_kernel(Kv4Args a, Kv4Batch b) {
  constexpr int RT = kKv4ChunkRows / 64;
  constexpr int PT = 4;  // tiles of 16 tokens whose scores are held at a time
  Kv4Work k;
  if (k.locate(a, b)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, q4 = lane >> 4;
  extern __shared__ __align__(16) uint8_t smem[];  // two pages
  const int row0 = k.rb * 64 * RT + 16 * RT * w;   // the wave's first row
  const bool rows = row0 < k.S.n * k.g;
  bf16x8 qf[RT][4];
  int lim[RT];
  float m[RT], l[RT];
  f32x4 o[RT][8];
#pragma unroll
  for (int c = 0; c < RT; ++c) {
    lim[c] = load_rows(qf[c], a, k, row0 + 16 * c + l16, q4);
    m[c] = -INFINITY, l[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[c][j] = f32x4{0, 0, 0, 0};
  }
  const int64_t all_see = k.first + k.rb * kKv4ChunkRows / k.g;  // every row of the block sees the positions up to here
  const int64_t none_see = k.first + min(row0 + 16 * RT - 1, k.S.n * k.g - 1) / k.g;  // and none those behind this
  const float sl = a.scale * kLog2e;
  const int32_t* table = a.table + (int64_t)k.S.seq * a.width;
  bool bad = k.bad;
  // Page p to LDS without registers, 1 KiB a load; the last is 768 bytes and zeros.
  auto load = [&](int p) {
    int id = table[p];
    if (id < 0 || id >= a.pages) bad = true, id = 0;
    const __amdgpu_buffer_rsrc_t r = buffer_rsrc(a.cache + ((int64_t)id * a.kv_heads + k.kh) * kRec, kRec);
    uint8_t* dst = smem + (p & 1) * kChunkBuf;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(dst + i * 4096 + w * 1024), 16,
                                               i * 4096 + w * 1024 + lane * 16, 0, 0, 0);
    if (w == 0)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(dst + kOffKs), 16, kOffKs + lane * 16, 0, 0, 0);
  };
  if (k.p0 < k.p1) load(k.p0);
  auto page = [&](int p, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    // This wave's loads have landed; then every wave's have, and every wave is done with the other buffer.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (p + 1 < k.p1) load(p + 1);
    const uint8_t* rec = smem + (p & 1) * kChunkBuf;
    if (!rows || (MASKED && (int64_t)p * kPage > none_see)) return;
    const uint2 ks = *reinterpret_cast<const uint2*>(rec + kOffKs + 128 * q4 + 8 * l16);
#pragma unroll
    for (int h0 = 0; h0 < 8; h0 += PT) {
      f32x4 st[RT][PT];  // S^T[16 (h0 + i) + 4 q4 + r][row]
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        const u32x4 kr = *reinterpret_cast<const u32x4*>(rec + (16 * (h0 + i) + l16) * 64 + 16 * q4);
        const float sc = __uint_as_float(((h0 + i < 4 ? ks.x : ks.y) >> (8 * ((h0 + i) & 3)) & 255u) << 23);
#pragma unroll
        for (int c = 0; c < RT; ++c) st[c][i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const bf16x8 ak = widen(kr[s], sc);
#pragma unroll
          for (int c = 0; c < RT; ++c) st[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ak, qf[c][s], st[c][i], 0, 0, 0);
        }
      }
      u32x4 vs[PT / 2];
#pragma unroll
      for (int i = 0; i < PT / 2; ++i) vs[i] = *reinterpret_cast<const u32x4*>(rec + kOffVs + 64 * q4 + 8 * h0 + 16 * i);
      uint2 vr[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) vr[j] = *reinterpret_cast<const uint2*>(rec + kOffV + (16 * j + l16) * 64 + 16 * q4 + 2 * h0);
      bf16x8 pw[RT][PT / 2];
      const int t0 = p * kPage + 16 * h0 + 4 * q4;
#pragma unroll
      for (int c = 0; c < RT; ++c) weigh<PT, MASKED>(st[c], pw[c], vs, sl, t0, lim[c], m[c], l[c], o[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int u = 0; u < PT / 2; ++u) {
          const bf16x8 av = widen(u ? vr[j].y : vr[j].x, 1.0f);
#pragma unroll
          for (int c = 0; c < RT; ++c) o[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, pw[c][u], o[c][j], 0, 0, 0);
        }
      }
    }
  };
  int p = k.p0;
  for (; p < k.p1 && (int64_t)p * kPage + kPage - 1 <= all_see; ++p) page(p, std::false_type{});
  for (; p < k.p1; ++p) page(p, std::true_type{});
  if (!rows) return;
#pragma unroll
  for (int c = 0; c < RT; ++c)
    write_rows(a, k, 16 * RT * w + 16 * c + l16, m[c], bad ? __uint_as_float(0x7FC00000u) : rows_sum(l[c]), o[c], q4);
}

// Joins the splits of a row in their order. W waves per (row, query head), each a range of the splits, two elements a lane,
// eight splits' loads on their way. Bound by memory where there are many rows (4 x 64 rows x 32 heads, up to 13 splits: 31 MB in
// 8.4 us), by latency otherwise (16 rows: 3.5 us). Four waves where the splits are many and the rows few, attention and
// join with one / four: one row of 32 heads, 16 splits 9.4 / 9.9, 64 splits 23.1 / 20.7; 8 heads, 128 splits 19.2 / 13.3; the 8192
// (row, head) above 46 / 58.
template <int W>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4Args a, Kv4Batch b, int64_t rows) {
  const int lane = threadIdx.x & 63, R = a.block_rows, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t at = (int64_t)blockIdx.x * (4 / W) + w / W;  // (row of the batch, head)
  if (W == 1 && at >= rows * a.heads) return;
  const int64_t row = b.s[0].row0 + at / a.heads;
  const int h = (int)(at % a.heads), g = a.heads / a.kv_heads;
  // rows of empty sequences do not exist, so the last sequence that begins at or before the row holds it
  const Kv4Seq S = b.same ? find_seq(b, (int)(row - b.s[0].row0) / b.same * b.wgs)
                          : b.s[__popcll(__ballot(lane < b.count && b.s[lane < b.count ? lane : 0].row0 <= row)) - 1];
  const int r = (int)(row - S.row0) * g + h % g;
  int64_t len = a.lengths[S.seq];
  if (len < 0 || len > a.max_length) len = 0;  // of a bad length the first split's sum is NaN
  const int used = (int)((len + kPage - 1) / kPage);
  const int ns = max(1, (used + a.chunk - 1) / a.chunk);
  const int64_t unit = ((int64_t)(S.blk0 + r / R) * a.kv_heads + h / g) * a.splits;
  float m = -INFINITY, l = 0.0f;
  float2 o = make_float2(0.0f, 0.0f);
  const int each = (ns + W - 1) / W, end = min(ns, (w % W + 1) * each);
  for (int s0 = w % W * each; s0 < end; s0 += 64) {  // a lane's factor is that of split s0 + lane
    const int n = __builtin_amdgcn_readfirstlane(min(64, end - s0));
    const int64_t u = (unit + s0) * R + r % R;
    const float2 ml = lane < n ? a.part_ml[u + (int64_t)lane * R] : make_float2(-INFINITY, 0.0f);
    const float mn = fmaxf(m, wave_max(ml.x)), ms = mn == -INFINITY ? 0.0f : mn;
    const float f = __builtin_amdgcn_exp2f(ml.x - ms), fa = __builtin_amdgcn_exp2f(m - ms);
    m = mn;
    l = l * fa + group_sum<64>(ml.y * f);
    o.x *= fa;
    o.y *= fa;
    for (int s = 0; s < n; s += 8) {
      float2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] = *reinterpret_cast<const float2*>(a.part + (u + (int64_t)min(s + i, n - 1) * R) * DH + 2 * lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // the factors of lanes past n are 0
        const float fs = s + i < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s + i)) : 0.0f;
        o.x = fmaf(x[i].x, fs, o.x);
        o.y = fmaf(x[i].y, fs, o.y);
      }
    }
  }
  if constexpr (W > 1) {
    __shared__ float2 ml[W], ox[W][64];
    if (lane == 0) ml[w] = make_float2(m, l);
    ox[w][lane] = o;
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int i = 1; i < W; ++i) m = fmaxf(m, ml[i].x);
    const float ms = m == -INFINITY ? 0.0f : m;
    l = 0.0f;
    o = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float f = __builtin_amdgcn_exp2f(ml[i].x - ms);
      l = fmaf(ml[i].y, f, l);
      o.x = fmaf(ox[i][lane].x, f, o.x);
      o.y = fmaf(ox[i][lane].y, f, o.y);
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (lane == 0) a.lse[(int64_t)h * a.N + row] = l == 0.0f ? -INFINITY : m / kLog2e + logf(l);
  *reinterpret_cast<uint32_t*>(a.o + (row * a.heads + h) * DH + 2 * lane) = pack_bf16x2(o.x * inv, o.y * inv);
}

hipError_t launch_kv4_append(const Kv4Args& a, Kv4Batch b, hipStream_t s) {
  int64_t n = 0;
  for (int i = 0; i < b.count; ++i) {
    b.s[i].wg_begin = (int32_t)n;
    if (b.s[i].n > 0) n += ((int64_t)((b.s[i].n + kPage - 2) / kPage + 1) * a.kv_heads + 7) / 8 * 32;
    if (i == 0) b.wgs = (int32_t)n;
  }
  if (n <= 0) return hipSuccess;
  KernelTimer t(K_KV4_APPEND, s);
  hipLaunchKernelGGL(kv4_append_kernel, dim3((unsigned)n), dim3(256), 0, s, a, b);
  return hipGetLastError();
}

template <class K>
static hipError_t launch_blocks(K kernel, LdsLimit& limit, size_t lds, const Kv4Args& a, Kv4Batch b, hipStream_t s) {
  if (lds)
    if (hipError_t e = limit.raise((const void*)kernel, lds)) return e;
  const int g = a.heads / a.kv_heads;
  int64_t n = 0, rows = 0;
  for (int i = 0; i < b.count; ++i) {
    const int64_t blocks = ((int64_t)b.s[i].n * g + a.block_rows - 1) / a.block_rows;
    b.s[i].wg_begin = (int32_t)n;
    n += blocks * a.kv_heads * a.splits;
    if (i == 0) b.wgs = (int32_t)n, b.blocks = (int32_t)blocks;
    rows += b.s[i].n;
  }
  if (n <= 0) return hipSuccess;
  {
    KernelTimer t(K_KV4_ATTN, s);
    hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(256), lds, s, a, b);
  }
  if (a.splits > 1) {
    KernelTimer t(K_KV4_JOIN, s);
    if (a.splits > 16 && rows * a.heads <= 1024)
      hipLaunchKernelGGL(kv4_join_kernel<4>, dim3((unsigned)(rows * a.heads)), dim3(256), 0, s, a, b, rows);
    else
      hipLaunchKernelGGL(kv4_join_kernel<1>, dim3((unsigned)((rows * a.heads + 3) / 4)), dim3(256), 0, s, a, b, rows);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_attention(const Kv4Args& a, const Kv4Batch& b, hipStream_t s) {
  static LdsLimit limits[2];
  return a.block_rows == 16 ? launch_blocks(kv4_decode_kernel, limits[0], 0, a, b, s)
                            : launch_blocks(kv4_chunk_kernel, limits[1], 2 * kChunkBuf, a, b, s);
}

}  // namespace attt

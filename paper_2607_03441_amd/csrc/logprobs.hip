// Log-probabilities of given tokens through the LM head, the entropy of each row's distribution, and its top
// alternatives (what the model that the update of Eq. 10 trains says about a text):
//   z = W h, lse = log sum_v exp(z_v), logp = z_y - lse, entropy = lse - sum_v p_v z_v,
//   the `top` largest z_v - lse with their ids, equal logits in the order of their ids.
// With m any reference, s = sum exp(z - m) and t = sum (z - m) exp(z - m): lse = m + log s and
// entropy = log s - t / s, which does not cancel where one token has nearly all the probability.
#include "common.hpp"
#include "gemm_core.hpp"
#include "internal.hpp"
#include "lds_limit.hpp"

namespace attt {

namespace {
// A logit and its id; better: larger, or as large with the lower id. (-inf, -1 as unsigned) is below every logit.
struct Cand {
  float z;
  uint32_t id;
};
__device__ __forceinline__ bool better(Cand a, Cand b) { return a.z > b.z || (a.z == b.z && a.id < b.id); }
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ Cand wave_best(Cand c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Cand x = {__shfl_xor(c.z, o, 64), (uint32_t)__shfl_xor((int)c.id, o, 64)};
    if (better(x, c)) c = x;
  }
  return c;
}

// Joins (m2, s2, t2) into (m, s, t). An empty side is (-inf, 0, 0).
__device__ __forceinline__ void stats_join(float& m, float& s, float& t, float m2, float s2, float t2) {
  const float mn = fmaxf(m, m2);
  if (mn == -INFINITY) {  // nothing finite yet: a NaN is kept
    s += s2;
    t += t2;
    return;
  }
  const float da = m - mn, db = m2 - mn, fa = expf(da), fb = expf(db);
  t = (m == -INFINITY ? t : fa * (t + da * s)) + (m2 == -INFINITY ? t2 : fb * (t2 + db * s2));
  s = (m == -INFINITY ? s : fa * s) + (m2 == -INFINITY ? s2 : fb * s2);
  m = mn;
}
}  // namespace

// Logits of 128 vocabulary entries x 128 rows, transposed as in the cross-entropy's forward: a lane holds
// groups of four consecutive entries of its row.
__global__ __launch_bounds__(256) void lp_logits_bf16_kernel(LpArgs a, int tiles_v, int tiles_t) {
  using C = CfgSmall;
  extern __shared__ __align__(16) uint8_t smem[];
  int tv, tt;
  tile_of(blockIdx.x, tiles_v, tiles_t, tv, tt);
  const int v0 = tv * C::BM, t0 = tt * C::BN;
  f32x16 acc[C::TM][C::TN];
  mfma_mainloop<C>(static_cast<const bf16_t*>(a.W) + (int64_t)v0 * a.d, a.d, a.V - v0,
                   static_cast<const bf16_t*>(a.h) + (int64_t)(a.row0 + t0) * a.d, a.d, a.rows - t0, a.d,
                   reinterpret_cast<bf16_t*>(smem), acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / C::WGN, wn = wave % C::WGN;
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int t = t0 + wn * C::WTN + j * 32 + (lane & 31);
    if (t >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int v = v0 + wm * C::WTM + i * 32 + mfma_row(r, lane);
        if (v < a.V)  // ldz is a multiple of 4: a group that begins inside the row ends in its padding
          *reinterpret_cast<f32x4*>(a.logits + (int64_t)t * a.ldz + v) =
              f32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
      }
  }
}

// The same in float32: 64 x 64 tiles on the float32 matrix instruction, K in steps of 32 through LDS.
__global__ __launch_bounds__(256) void lp_logits_f32_kernel(LpArgs a, int tiles_t) {
  constexpr int T = 64, K = 32, P = K + 4;
  __shared__ __align__(16) float lds[2][2][T * P];
  const int t0 = (int)(blockIdx.x % tiles_t) * T, v0 = (int)(blockIdx.x / tiles_t) * T;
  const float* A = static_cast<const float*>(a.W) + (int64_t)v0 * a.d;
  const float* B = static_cast<const float*>(a.h) + (int64_t)(a.row0 + t0) * a.d;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31, hi = lane >> 5;
  const int lr = tid >> 3, lk = (tid & 7) * 4;
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
  f32x4 ra[2], rb[2];
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = lr + 32 * u;
      const bool kin = k0 + lk < a.d;
      ra[u] = kin && v0 + row < a.V ? *reinterpret_cast<const f32x4*>(A + (int64_t)row * a.d + k0 + lk) : f32x4{0, 0, 0, 0};
      rb[u] = kin && t0 + row < a.rows ? *reinterpret_cast<const f32x4*>(B + (int64_t)row * a.d + k0 + lk) : f32x4{0, 0, 0, 0};
    }
  };
  load(0);
  int buf = 0;
  for (int k0 = 0; k0 < a.d; k0 += K, buf ^= 1) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      *reinterpret_cast<f32x4*>(&lds[buf][0][(lr + 32 * u) * P + lk]) = ra[u];
      *reinterpret_cast<f32x4*>(&lds[buf][1][(lr + 32 * u) * P + lk]) = rb[u];
    }
    // this step's tiles are stored; the other buffer's readers passed the barrier before it is stored again
    __syncthreads();
    if (k0 + K < a.d) load(k0 + K);
    const float* As = &lds[buf][0][(wm * 32 + l32) * P + 4 * hi];
    const float* Bs = &lds[buf][1][(wn * 32 + l32) * P + 4 * hi];
#pragma unroll
    for (int j = 0; j < K / 8; ++j) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(As + 8 * j), y = *reinterpret_cast<const f32x4*>(Bs + 8 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
    }
  }
  const int t = t0 + wn * 32 + l32;
  if (t >= a.rows) return;
#pragma unroll
  for (int r = 0; r < 16; r += 4) {
    const int v = v0 + wm * 32 + mfma_row(r, lane);
    if (v < a.V)
      *reinterpret_cast<f32x4*>(a.logits + (int64_t)t * a.ldz + v) = f32x4{acc[r], acc[r + 1], acc[r + 2], acc[r + 3]};
  }
}

// The logits of a row tile of 256 tokens without memory for them: a persistent workgroup walks the vocabulary tiles split,
// split + splits, ... of the product z^T = W h^T (gemm_core.hpp's 256 x 256 tiles on eight waves) and takes what it
// needs from each while the next tile's first loads are on their way. A lane holds 32 logits of each of 4 tokens.
// Statistics: every token's (m, s, t) per half of the tile's rows (wave row), kept in LDS.
// Alternatives: a token's list of the best so far lies in its place of `lists`, the last of it as a threshold in LDS.
// A tile's logits above the threshold are handed to the token's thread through kHand places in LDS, in as
// many rounds as it takes; that thread sorts them into the list and raises the threshold. After the first tile
// there are few: a tile of M replaces about top / M of them. Ids grow from tile to tile, so that a logit equal to the
// threshold never displaces an earlier one; within a tile the ids decide. The list does not depend on
// the order in which candidates arrive.
constexpr int kHand = 8;
struct LpFusedLds {
  float m[2][256], s[2][256], t[2][256];
  float zy[256];        // the label's logit; NaN until it has been met
  int32_t y[256];       // the label; negative: none in the vocabulary
  float thr[256];       // the list's last logit; NaN: the list is not full; +inf: no list
  uint32_t thr_id[256]; // and its id
  int32_t count[256];   // candidates of the round, kHand of which have a place
  Cand hand[256][kHand];
};
constexpr size_t kLpFusedLds = CfgBig::LDS + sizeof(LpFusedLds);
static_assert(kLpFusedLds <= 160 * 1024, "LDS");

// KB: places of a list (0: no alternatives)
template <int KB>
__global__ __launch_bounds__(512) void lp_fused_kernel(LpArgs a, int tiles_t, int tiles_v) {
  using C = CfgBig;
  extern __shared__ __align__(16) uint8_t smem[];
  bf16_t* stages = reinterpret_cast<bf16_t*>(smem);
  LpFusedLds& L = *reinterpret_cast<LpFusedLds*>(smem + C::LDS);
  const int tid = threadIdx.x;
  int tt, split;
  tile_of(blockIdx.x, tiles_t, a.splits, tt, split);
  const int t0 = tt * 256, nt = min(256, a.rows - t0);
  if (tid < 256) {
    L.m[0][tid] = L.m[1][tid] = -INFINITY;
    L.s[0][tid] = L.s[1][tid] = L.t[0][tid] = L.t[1][tid] = 0.0f;
    L.zy[tid] = __uint_as_float(0x7FC00000u);
    const int y = tid < nt ? a.labels[a.row0 + t0 + tid] : -1;
    L.y[tid] = y < a.V ? y : -1;
    L.thr[tid] = tid < nt ? __uint_as_float(0x7FC00000u) : INFINITY;
    L.thr_id[tid] = kNone;
    L.count[tid] = 0;
  }
  const bf16_t* W = static_cast<const bf16_t*>(a.W);
  const bf16_t* h = static_cast<const bf16_t*>(a.h) + (int64_t)(a.row0 + t0) * a.d;
  auto prologue = [&](int tv, int id) {
    mfma_pp_prologue<C>(W + (int64_t)tv * 256 * a.d, a.d, a.V - tv * 256, h, a.d, nt, a.d, stages, id);
  };
  prologue(split, tid);
  bool first = true;
  for (int tv = split; tv < tiles_v; tv += a.splits, first = false) {
    int id = tid;
    asm volatile("" : "+v"(id));  // what is derived from it is not kept across the mainloop
    const int v0 = tv * 256;
    Acc16 acc;
    mfma_mainloop_pp16<C>(W + (int64_t)v0 * a.d, a.d, a.V - v0, h, a.d, nt, a.d, stages, acc, id, true);
    if (tv + a.splits < tiles_v) prologue(tv + a.splits, id);
    const int lane = id & 63, w = __builtin_amdgcn_readfirstlane(id >> 6);
    const int wm = w >> 2, l16 = lane & 15, q4 = lane >> 4;
    const int vb = v0 + wm * 128 + 4 * q4;  // entry (i, r) of the lane: vb + 16 i + r
    uint32_t pending[Mma16::TN];            // bit 4 i + r
    const bool whole = v0 + 256 <= a.V;
#pragma unroll
    for (int j = 0; j < Mma16::TN; ++j) {
      const int tok = (w & 3) * 64 + 16 * j + l16;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (vb + 16 * i + r >= a.V) acc[i][j][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, acc[i][j][r]);
      const float m_old = L.m[wm][tok], m = fmaxf(m_old, rows_max(mx));
      const float m0 = m == -INFINITY ? 0.0f : m;
      const float mb = m0 * kLog2e;
      float s = 0.0f, t = 0.0f;
#pragma unroll
      for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], kLog2e, -mb));
          s += e;
          t = fmaf(fmaxf(acc[i][j][r] - m0, -200.0f), e, t);  // e is 0 there: -inf times it would not be
        }
      s = rows_sum(s);
      t = rows_sum(t);
      const float s_old = L.s[wm][tok], t_old = L.t[wm][tok];
      const float dm = m_old == -INFINITY ? 0.0f : m_old - m0, f = __builtin_amdgcn_exp2f(dm * kLog2e);
      const int y = L.y[tok] - (v0 + wm * 128);
      const bool has = y >= 0 && y < 128 && (y >> 2 & 3) == q4;
      if (__any(has)) {
        const int e = (y >> 4) * 4 + (y & 3);
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (e == 4 * i + r) z = acc[i][j][r];
        if (has) L.zy[tok] = z;
      }
      // all of the wave's reads of the token's old values come before the writes
      if (q4 == 0) {
        L.m[wm][tok] = m;
        L.s[wm][tok] = s_old * f + s;
        L.t[wm][tok] = (t_old + dm * s_old) * f + t;
      }
      if constexpr (KB > 0) {
        const float thr = L.thr[tok];
        uint32_t p = 0;
#pragma unroll
        for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(acc[i][j][r] <= thr) && (whole || vb + 16 * i + r < a.V)) p |= 1u << (4 * i + r);
        pending[j] = p;
      }
    }
    if constexpr (KB > 0) {
      for (;;) {
#pragma unroll
        for (int j = 0; j < Mma16::TN; ++j) {
          const int tok = (w & 3) * 64 + 16 * j + l16;
          if (pending[j]) {
#pragma unroll
            for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (pending[j] >> (4 * i + r) & 1) {
                  const int at = atomicAdd(&L.count[tok], 1);
                  if (at < kHand) {
                    L.hand[tok][at] = {acc[i][j][r], (uint32_t)(vb + 16 * i + r)};
                    pending[j] &= ~(1u << (4 * i + r));
                  }
                }
          }
        }
        __syncthreads();
        bool more = false;
        const int n = id < 256 ? L.count[id] : 0;
        if (n > 0) {
          more = n > kHand;
          Cand list[KB];
          float2* mine = a.lists + ((int64_t)(t0 + id) * a.splits + split) * KB;
          const bool fresh = first && L.thr_id[id] == kNone;  // nothing has been written yet
#pragma unroll
          for (int k = 0; k < KB; ++k) {
            const float2 x = fresh ? make_float2(-INFINITY, __uint_as_float(kNone)) : mine[k];
            list[k] = {x.x, __float_as_uint(x.y)};
          }
          bool nan = false;
#pragma unroll 1
          for (int c = 0; c < min(n, kHand); ++c) {
            Cand x = L.hand[id][c];
            nan |= x.z != x.z;
#pragma unroll
            for (int k = 0; k < KB; ++k) {
              const bool up = better(x, list[k]);
              const Cand y = up ? list[k] : x;
              list[k] = up ? x : list[k];
              x = y;
            }
          }
          Cand last = list[0];
#pragma unroll
          for (int k = 0; k < KB; ++k) {
            mine[k] = make_float2(list[k].z, __uint_as_float(list[k].id));
            if (k == a.top - 1) last = list[k];
          }
          // an id marks the list as written even while it is not full
          L.thr[id] = nan ? INFINITY : last.id == kNone ? __uint_as_float(0x7FC00000u) : last.z;
          L.thr_id[id] = last.id == kNone ? kNone - 1 : last.id;
          L.count[id] = 0;
        }
        if (!__syncthreads_or(more)) break;
#pragma unroll
        for (int j = 0; j < Mma16::TN; ++j) {
          const int tok = (w & 3) * 64 + 16 * j + l16;
          const float thr = L.thr[tok];
          const uint32_t ti = L.thr_id[tok];
#pragma unroll
          for (int i = 0; i < Mma16::TM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (acc[i][j][r] < thr || (acc[i][j][r] == thr && (uint32_t)(vb + 16 * i + r) > ti)) pending[j] &= ~(1u << (4 * i + r));
        }
      }
    }
  }
  __syncthreads();
  if (tid < nt) {
    float m = L.m[0][tid], s = L.s[0][tid], t = L.t[0][tid];
    stats_join(m, s, t, L.m[1][tid], L.s[1][tid], L.t[1][tid]);
    const int64_t at = (int64_t)(t0 + tid) * a.splits + split;
    a.stats[at] = make_float4(m, s, t, L.zy[tid]);
    if constexpr (KB > 0)
      if (L.thr_id[tid] == kNone)  // not one candidate
        for (int k = 0; k < KB; ++k) a.lists[at * KB + k] = make_float2(-INFINITY, __uint_as_float(kNone));
  }
}

// Statistics and the best `top` of kLpRowChunk logits of one staged row: 16 a thread, in registers. The best
// are drawn one after the other: the best of each thread's, of each wave's, of the workgroup's.
__global__ __launch_bounds__(256) void lp_rows_kernel(LpArgs a) {
  constexpr int E = kLpRowChunk / 256;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const float* z = a.logits + (int64_t)row * a.ldz;
  const int v0 = split * kLpRowChunk;
  float x[E];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; i += 4) {
    const int v = v0 + (i / 4 * 256 + tid) * 4;
    f32x4 y = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (v < a.V) y = *reinterpret_cast<const f32x4*>(z + v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[i + e] = v + e < a.V ? y[e] : -INFINITY;
      m = fmaxf(m, x[i + e]);
    }
  }
  float s = 0.0f, t = 0.0f;
  const float m0 = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x[i] - m0, e = expf(d);
    s += e;
    t += e == 0.0f ? 0.0f : d * e;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) stats_join(m, s, t, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64), __shfl_xor(t, o, 64));
  __shared__ float4 st[4];
  __shared__ Cand best[2][4];
  if (lane == 0) st[w] = make_float4(m, s, t, 0.0f);
  __syncthreads();
  const int64_t at = (int64_t)row * a.splits + split;
  if (tid == 0) {
    for (int i = 1; i < 4; ++i) stats_join(m, s, t, st[i].x, st[i].y, st[i].z);
    const int y = a.labels[a.row0 + row];
    a.stats[at] = make_float4(m, s, t, y >= v0 && y < min(a.V, v0 + kLpRowChunk) ? z[y] : __uint_as_float(0x7FC00000u));
  }
  uint32_t taken = 0;
  auto mine = [&]() {
    Cand c = {-INFINITY, kNone};
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int v = v0 + (i / 4 * 256 + tid) * 4 + (i & 3);
      const Cand k = {x[i], (uint32_t)v};
      if (v < a.V && !(taken >> i & 1) && better(k, c)) c = k;
    }
    return c;
  };
  Cand c = a.top > 0 ? mine() : Cand{};
  for (int n = 0; n < a.top; ++n) {
    const Cand wb = wave_best(c);
    if (lane == 0) best[n & 1][w] = wb;
    __syncthreads();
    Cand b = best[n & 1][0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (better(best[n & 1][i], b)) b = best[n & 1][i];
    if (tid == 0) a.lists[at * a.places + n] = make_float2(b.z, __uint_as_float(b.id));
    if (b.id != kNone && b.id == c.id) {
      const int rel = (int)b.id - v0;
      taken |= 1u << (rel / 1024 * 4 + (rel & 3));
      c = mine();
    }
  }
}

// Joins a row's splits and writes its results. One wave per row.
__global__ __launch_bounds__(256) void lp_join_kernel(LpArgs a) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const int64_t at = (int64_t)row * a.splits, out = a.row0 + row;
  float m = -INFINITY, s = 0.0f, t = 0.0f, zy = __uint_as_float(0x7FC00000u);
  for (int i = lane; i < a.splits; i += 64) {
    const float4 x = a.stats[at + i];
    stats_join(m, s, t, x.x, x.y, x.z);
    if (x.w == x.w) zy = x.w;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    stats_join(m, s, t, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64), __shfl_xor(t, o, 64));
    const float other = __shfl_xor(zy, o, 64);
    if (other == other) zy = other;
  }
  const float ls = logf(s), lse = m + ls;
  if (lane == 0) {
    a.logp[out] = zy - lse;
    if (a.entropy) a.entropy[out] = ls - t / s;
  }
  // the best of the lists, one after the other; a row that has no finite lse has none
  const int n = a.splits * a.top;
  Cand last = {INFINITY, 0};
  bool first = true;
  for (int k = 0; k < a.top; ++k) {
    Cand c = {-INFINITY, kNone};
    for (int i = lane; i < n; i += 64) {
      const float2 x = a.lists[(at + i / a.top) * a.places + i % a.top];
      const Cand y = {x.x, __float_as_uint(x.y)};
      if (y.id != kNone && (first || better(last, y)) && better(y, c)) c = y;
    }
    c = wave_best(c);
    last = c;
    first = false;
    if (lane == 0) {
      const bool ok = __builtin_isfinite(lse) && c.id != kNone;
      a.top_ids[out * a.top + k] = ok ? (int32_t)c.id : -1;
      a.top_logp[out * a.top + k] = ok ? c.z - lse : __uint_as_float(0x7FC00000u);
    }
  }
}

hipError_t launch_lp_logits(int dtype, const LpArgs& a, hipStream_t s) {
  KernelTimer t(K_LP_LOGITS, s);
  if (dtype == 1) {
    static LdsLimit limit;
    if (hipError_t e = limit.raise((const void*)lp_logits_bf16_kernel, CfgSmall::LDS)) return e;
    const int tv = (a.V + CfgSmall::BM - 1) / CfgSmall::BM, tt = (a.rows + CfgSmall::BN - 1) / CfgSmall::BN;
    hipLaunchKernelGGL(lp_logits_bf16_kernel, dim3(tv * tt), dim3(256), CfgSmall::LDS, s, a, tv, tt);
  } else {
    const int tv = (a.V + 63) / 64, tt = (a.rows + 63) / 64;
    hipLaunchKernelGGL(lp_logits_f32_kernel, dim3(tv * tt), dim3(256), 0, s, a, tt);
  }
  return hipGetLastError();
}

template <int KB>
static hipError_t launch_fused(const LpArgs& a, hipStream_t s) {
  static LdsLimit limit;
  if (hipError_t e = limit.raise((const void*)lp_fused_kernel<KB>, kLpFusedLds)) return e;
  const int tiles_t = (a.rows + 255) / 256, tiles_v = (a.V + 255) / 256;
  KernelTimer t(K_LP_FUSED, s);
  hipLaunchKernelGGL(lp_fused_kernel<KB>, dim3(tiles_t * a.splits), dim3(512), kLpFusedLds, s, a, tiles_t, tiles_v);
  return hipGetLastError();
}

hipError_t launch_lp_fused(const LpArgs& a, hipStream_t s) {
  return a.top == 0 ? launch_fused<0>(a, s) : a.places == 8 ? launch_fused<8>(a, s) : a.places == 16 ? launch_fused<16>(a, s) : launch_fused<32>(a, s);
}

hipError_t launch_lp_rows(const LpArgs& a, hipStream_t s) {
  KernelTimer t(K_LP_ROWS, s);
  hipLaunchKernelGGL(lp_rows_kernel, dim3((unsigned)a.rows * a.splits), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_lp_join(const LpArgs& a, hipStream_t s) {
  KernelTimer t(K_LP_JOIN, s);
  hipLaunchKernelGGL(lp_join_kernel, dim3((a.rows + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace attt

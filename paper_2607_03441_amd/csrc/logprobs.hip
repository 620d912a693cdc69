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
    if (tid == 0) a.lists[at * a.top + n] = make_float2(b.z, __uint_as_float(b.id));
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
      const float2 x = a.lists[at * a.top + i];
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

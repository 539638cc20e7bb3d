// Balance loss of a router over its experts, with per-expert counts, a z loss
// and the gradient of the logits (unif_moe_balance_loss). With p = softmax(z_t)
// of each of the n valid tokens, c_j the number of times expert j is selected:
//   f_j = c_j / sum c,  P_j = sum_t p_tj / n
//   balance = K sum_j f_j P_j,  zloss = sum_t lse(z_t)^2 / n
//   loss = w_b balance + w_z zloss
//   dloss/dz_tj = p_tj / n (w_b K (f_j - sum_i f_i p_ti) + 2 w_z lse(z_t))
//
// The gradient needs the counts of all tokens, so there are two kernels: the
// first leaves each CTA's sums in the workspace, the second adds them (in the
// CTAs' order: results do not change from run to run) and writes the gradient
// from a second reading of the logits, which the first left in L2.
// A token belongs to L lanes of a warp, which hold E logits each.
#include <cuda_bf16.h>
#include <math.h>

#include "internal.cuh"

namespace unif {
namespace balance {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Args {
  int T, K, n_q;
  const void* logits;
  long long ld, ld_q;
  const int32_t* q;
  const int32_t* k;
  const uint8_t* mask;
  float w_b, w_z;
  float* loss;      // [3]
  int32_t* counts;  // [K]
  float* prob;      // [K]
  float* dlogits;   // [T][K] or NULL
  float* part_p;    // [CTAs][K]
  int32_t* part_c;  // [CTAs][K]
  float* part_z;    // [CTAs]
  int32_t* part_n;  // [CTAs]
  int ctas;         // of the first kernel
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

template <int L>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// exp(z - max) of a token's logits in e (0 past K), their sum and the maximum;
// false for padding and for a token whose logits are all -inf.
template <typename T, int L, int E>
__device__ __forceinline__ bool softmax(const Args& a, int t, int lane, float (&e)[E], float& top,
                                        float& sum) {
  const bool in = t < a.T && (!a.mask || a.mask[t]);
  const T* z = static_cast<const T*>(a.logits) + (long long)t * a.ld;
  top = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int c = i * L + lane;
    e[i] = in && c < a.K ? to_float(z[c]) : -INFINITY;
    top = fmaxf(top, e[i]);
  }
  top = lanes_max<L>(top);
  const float base = top == -INFINITY ? 0.f : top;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    e[i] = __expf(e[i] - base);
    sum += e[i];
  }
  sum = lanes_sum<L>(sum);
  return in && (top != -INFINITY || isnan(sum));
}

template <typename T, int L, int E>
__global__ void __launch_bounds__(kThreads) sums_kernel(const Args a) {
  extern __shared__ float sh[];  // [kWarps][K] probabilities, then [K] counts
  __shared__ float z_sh[kWarps];
  __shared__ int n_sh[kWarps];
  int* cnt = reinterpret_cast<int*>(sh + kWarps * a.K);
  for (int i = threadIdx.x; i < a.K; i += kThreads) cnt[i] = 0;
  __syncthreads();
  constexpr int kTok = kThreads / L;  // tokens of a CTA at a time
  const int lane = threadIdx.x % L, tok = threadIdx.x / L, warp = threadIdx.x / 32;
  float p[E], zs = 0.f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) p[i] = 0.f;
  for (long long base = (long long)blockIdx.x * kTok; base < a.T; base += (long long)gridDim.x * kTok) {
    const long long tt = base + tok;
    const int t = (int)min(tt, (long long)a.T);
    float e[E], top, sum;
    const bool valid = softmax<T, L, E>(a, t, lane, e, top, sum);
    if (valid) {
      const float inv = 1.f / sum, lse = top + logf(sum);
#pragma unroll
      for (int i = 0; i < E; ++i) p[i] = fmaf(e[i], inv, p[i]);
      if (lane == 0) {
        zs = fmaf(lse, lse, zs);
        ++n;
      }
      int m = a.n_q;
      if (a.k) m = min(m, a.k[t]);
      for (int i = lane; i < m; i += L) {
        const int j = a.q[(long long)t * a.ld_q + i];
        if (j >= 0 && j < a.K) atomicAdd(&cnt[j], 1);
      }
    }
  }
  // the groups of a warp, then the warps, in a fixed order
#pragma unroll
  for (int i = 0; i < E; ++i) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) p[i] += __shfl_xor_sync(0xffffffffu, p[i], o);
    const int c = i * L + lane;
    if ((threadIdx.x & 31) < L && c < a.K) sh[warp * a.K + c] = p[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    zs += __shfl_xor_sync(0xffffffffu, zs, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if ((threadIdx.x & 31) == 0) {
    z_sh[warp] = zs;
    n_sh[warp] = n;
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.K; c += kThreads) {
    float s = 0.f;
    for (int w = 0; w < kWarps; ++w) s += sh[w * a.K + c];
    a.part_p[(long long)blockIdx.x * a.K + c] = s;
    a.part_c[(long long)blockIdx.x * a.K + c] = cnt[c];
  }
  if (threadIdx.x == 0) {
    float s = 0.f;
    int m = 0;
    for (int w = 0; w < kWarps; ++w) { s += z_sh[w]; m += n_sh[w]; }
    a.part_z[blockIdx.x] = s;
    a.part_n[blockIdx.x] = m;
  }
}

template <typename T, int L, int E>
__global__ void __launch_bounds__(kThreads) gradient_kernel(const Args a) {
  extern __shared__ float sh[];  // [K] f, then [kWarps][K] shares of the sums
  __shared__ int all[2];
  __shared__ float fl[kWarps];
  float* f = sh;
  int* share = reinterpret_cast<int*>(sh + a.K);
  float* share_p = sh + a.K;
  const int lane32 = threadIdx.x & 31, warp = threadIdx.x / 32;
  if (threadIdx.x < 2) all[threadIdx.x] = 0;
  grid_dep_wait();
  // counts: whole numbers, so any order gives the same
  int sum_c = 0, n = 0;
  for (int c = lane32; c < a.K; c += 32) {
    int s = 0;
    for (int i = warp; i < a.ctas; i += kWarps) s += a.part_c[(long long)i * a.K + c];
    share[warp * a.K + c] = s;
    sum_c += s;
  }
  for (int i = threadIdx.x; i < a.ctas; i += kThreads) n += a.part_n[i];
  __syncthreads();
  atomicAdd(&all[0], sum_c);
  atomicAdd(&all[1], n);
  __syncthreads();
  const float inv_c = 1.f / (float)max(all[0], 1), inv_n = 1.f / (float)max(all[1], 1);
  for (int c = threadIdx.x; c < a.K; c += kThreads) {
    int s = 0;
    for (int w = 0; w < kWarps; ++w) s += share[w * a.K + c];
    f[c] = (float)s * inv_c;
    if (blockIdx.x == 0) a.counts[c] = s;
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int c = lane32; c < a.K; c += 32) {
      float s = 0.f;
      for (int i = warp; i < a.ctas; i += kWarps) s += a.part_p[(long long)i * a.K + c];
      share_p[warp * a.K + c] = s;
    }
    __syncthreads();
    float b = 0.f;
    for (int c = threadIdx.x; c < a.K; c += kThreads) {
      float s = 0.f;
      for (int w = 0; w < kWarps; ++w) s += share_p[w * a.K + c];
      s *= inv_n;
      a.prob[c] = s;
      b = fmaf(f[c], s, b);
    }
    b = lanes_sum<32>(b);
    if (lane32 == 0) fl[warp] = b;
    __syncthreads();
    if (warp == 0) {
      float z = 0.f;
      for (int i = lane32; i < a.ctas; i += 32) z += a.part_z[i];
      z = lanes_sum<32>(z) * inv_n;
      b = 0.f;
      for (int w = 0; w < kWarps; ++w) b += fl[w];
      b *= (float)a.K;
      if (lane32 == 0) {
        a.loss[0] = fmaf(a.w_b, b, a.w_z * z);
        a.loss[1] = b;
        a.loss[2] = z;
      }
    }
  }
  if (!a.dlogits) return;
  constexpr int kTok = kThreads / L;
  const int lane = threadIdx.x % L, tok = threadIdx.x / L;
  const float wb = a.w_b * (float)a.K, wz = 2.f * a.w_z;
  float fr[E];
#pragma unroll
  for (int i = 0; i < E; ++i) fr[i] = i * L + lane < a.K ? f[i * L + lane] : 0.f;
  for (long long base = (long long)blockIdx.x * kTok; base < a.T; base += (long long)gridDim.x * kTok) {
    const long long tt = base + tok;
    const int t = (int)min(tt, (long long)a.T);
    float e[E], top, sum;
    const bool valid = softmax<T, L, E>(a, t, lane, e, top, sum);
    const float inv = 1.f / sum;
    float fp = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      e[i] *= inv;
      fp = fmaf(fr[i], e[i], fp);
    }
    fp = lanes_sum<L>(fp);
    const float g = fmaf(wz, top + logf(sum), -wb * fp);
    if (tt < a.T)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int c = i * L + lane;
        if (c < a.K)
          a.dlogits[(long long)t * a.K + c] = valid ? e[i] * inv_n * fmaf(wb, fr[i], g) : 0.f;
      }
  }
}

int tokens_per_cta(int K) {
  const int lanes = K <= 4 ? 1 : K <= 8 ? 2 : K <= 16 ? 4 : K <= 32 ? 8 : K <= 64 ? 16 : 32;
  return kThreads / lanes;
}

// CTAs of both kernels: one per 256 lanes of tokens, at most two per SM.
int cta_count(int T, int K, int sms) {
  const long long want = ((long long)T + tokens_per_cta(K) - 1) / tokens_per_cta(K);
  return (int)(want < 1 ? 1 : want > 2ll * sms ? 2 * sms : want);
}

template <typename T, int L, int E>
cudaError_t launch_as(const Args& a, cudaStream_t s) {
  const size_t smem = (size_t)(kWarps + 1) * a.K * sizeof(float);
  sums_kernel<T, L, E><<<a.ctas, kThreads, smem, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_dependent(gradient_kernel<T, L, E>, dim3(a.dlogits ? a.ctas : 1), dim3(kThreads),
                          smem, s, a);
}

template <typename T>
cudaError_t launch(const Args& a, cudaStream_t s) {
  if (a.K <= 4) return launch_as<T, 1, 4>(a, s);
  if (a.K <= 8) return launch_as<T, 2, 4>(a, s);
  if (a.K <= 16) return launch_as<T, 4, 4>(a, s);
  if (a.K <= 32) return launch_as<T, 8, 4>(a, s);
  if (a.K <= 64) return launch_as<T, 16, 4>(a, s);
  if (a.K <= 128) return launch_as<T, 32, 4>(a, s);
  if (a.K <= 256) return launch_as<T, 32, 8>(a, s);
  return launch_as<T, 32, 16>(a, s);
}

// Offsets of the workspace's parts, each at a multiple of 16 bytes.
int64_t layout(int K, int ctas, int64_t (&at)[4]) {
  const int64_t row = ((int64_t)ctas * K * 4 + 15) / 16 * 16, one = ((int64_t)ctas * 4 + 15) / 16 * 16;
  at[0] = 0;
  at[1] = row;
  at[2] = 2 * row;
  at[3] = 2 * row + one;
  return 2 * row + 2 * one;
}

int sizes_ok(int T, int K) {
  if (T < 0 || K < 1) {
    set_error("bad sizes: T=%d K=%d", T, K);
    return UNIF_MOE_ERR_ARG;
  }
  if (K > UNIF_MOE_BALANCE_MAX_EXPERTS) {
    set_error("K=%d above %d", K, UNIF_MOE_BALANCE_MAX_EXPERTS);
    return UNIF_MOE_ERR_SHAPE;
  }
  return UNIF_MOE_OK;
}

}  // namespace balance
}  // namespace unif

using unif::set_error;
namespace bl = unif::balance;

extern "C" {

int64_t unif_moe_balance_workspace(int T, int K) {
  set_error("%s", "");
  if (bl::sizes_ok(T, K) != UNIF_MOE_OK) return -1;
  int sms = 0;
  if (unif::sm_count(&sms) != UNIF_MOE_OK) return -1;
  int64_t at[4];
  return bl::layout(K, bl::cta_count(T, K, sms), at);
}

int unif_moe_balance_loss(int T, int K, const void* logits, unif_moe_dtype dtype, int64_t ld,
                          const int32_t* q, int n_q, int64_t ld_q, const int32_t* k,
                          const uint8_t* mask, float w_balance, float w_z, float* loss,
                          int32_t* counts, float* prob, float* dlogits, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  set_error("%s", "");
  const int rc = bl::sizes_ok(T, K);
  if (rc != UNIF_MOE_OK) return rc;
  if (dtype != UNIF_MOE_F32 && dtype != UNIF_MOE_BF16) { set_error("bad dtype"); return UNIF_MOE_ERR_ARG; }
  if (!loss || !counts || !prob || (T > 0 && (!logits || (n_q > 0 && !q)))) {
    set_error("logits, q, loss, counts or prob is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (n_q < 0 || (T > 0 && (ld < K || ld_q < n_q))) {
    set_error("n_q=%d is negative, or a row stride (%lld, %lld) is below the row", n_q,
              (long long)ld, (long long)ld_q);
    return UNIF_MOE_ERR_ARG;
  }
  if (!isfinite(w_balance) || !isfinite(w_z)) {
    set_error("the weights of the losses must be finite");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  bl::Args a{};
  a.ctas = bl::cta_count(T, K, sms);
  int64_t at[4];
  const int64_t need = bl::layout(K, a.ctas, at);
  if (!workspace || workspace_bytes < need) {
    set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (reinterpret_cast<uintptr_t>(workspace) & 15u) {
    set_error("the workspace must be 16-byte aligned");
    return UNIF_MOE_ERR_ARG;
  }
  char* ws = static_cast<char*>(workspace);
  a.T = T; a.K = K; a.n_q = n_q; a.logits = logits; a.ld = ld; a.ld_q = ld_q; a.q = q; a.k = k;
  a.mask = mask; a.w_b = w_balance; a.w_z = w_z; a.loss = loss; a.counts = counts; a.prob = prob;
  a.dlogits = T > 0 ? dlogits : nullptr;
  a.part_p = reinterpret_cast<float*>(ws + at[0]);
  a.part_c = reinterpret_cast<int32_t*>(ws + at[1]);
  a.part_z = reinterpret_cast<float*>(ws + at[2]);
  a.part_n = reinterpret_cast<int32_t*>(ws + at[3]);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == UNIF_MOE_BF16 ? bl::launch<__nv_bfloat16>(a, s) : bl::launch<float>(a, s);
  if (e != cudaSuccess) {
    set_error("balance loss: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

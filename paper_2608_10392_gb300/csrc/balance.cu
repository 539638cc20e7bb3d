// Balance loss of a router over its experts, with per-expert counts, a z loss
// and the gradient of the logits (unif_moe_balance_loss). With p = softmax(z_t)
// of each of the n valid tokens, c_j the number of times expert j is selected:
//   f_j = c_j / sum c,  P_j = sum_t p_tj / n
//   balance = K sum_j f_j P_j,  zloss = sum_t lse(z_t)^2 / n
//   loss = w_b balance + w_z zloss
//   dloss/dz_tj = p_tj / n (w_b K (f_j - sum_i f_i p_ti) + 2 w_z lse(z_t))
//
// The gradient needs the counts of all tokens. Where a cluster of CTAs holds all
// of them at once, one kernel does it; otherwise there are two: the
// first leaves each CTA's sums in the workspace, the second adds them (in the
// CTAs' order: results do not change from run to run) and writes the gradient
// from a second reading of the logits, which the first left in L2.
// Latency bounds the call (us on the GPU, logits not in L2): 256 tokens of 4 experts 4.9,
// 12,608 of 8 8.6, both in one kernel; 65,536 of 32 in two 16.0, where the bytes need 2.6.
// A token belongs to L lanes of a warp, which hold E logits each. At most one CTA
// per SM: with two of 256 threads and one token of each group at a time, 65,536
// tokens of 32 experts took 17 and 21 us.
#include <cuda_bf16.h>
#include <math.h>

#include "internal.cuh"
#include "per_device.h"

namespace unif {
namespace balance {

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
  float* part_p;    // [K][CTAs]
  int32_t* part_c;  // [K][CTAs]
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

// Counts beyond 32 bits are added in two parts, the low 16 bits and the rest (counts
// below 2^48): shared memory adds no 64-bit numbers but in a loop that compares and tries
// again (65,536 tokens of 32 experts 16.4 us with those, 16.0 so).
struct Total {
  unsigned low, high;
  __device__ __forceinline__ void clear() { low = high = 0u; }
  __device__ __forceinline__ void add(long long c) {  // by any thread, in shared memory
    atomicAdd(&low, (unsigned)c & 0xffffu);
    atomicAdd(&high, (unsigned)(c >> 16));
  }
  __device__ __forceinline__ long long get() const { return ((long long)high << 16) + low; }
};
__device__ __forceinline__ long long warp_total(long long c) {
  const unsigned low = __reduce_add_sync(0xffffffffu, (unsigned)c & 0xffffu);
  return ((long long)__reduce_add_sync(0xffffffffu, (unsigned)(c >> 16)) << 16) + low;
}
// A count as it is given to the caller.
__device__ __forceinline__ int count32(long long c) { return (int)min(c, 0x7fffffffll); }

// Lane `lane` of a token's L lanes holds the columns lane E .. lane E + E - 1.
template <typename T, int L, int E, bool VEC>
__device__ __forceinline__ void load(const Args& a, bool in, int t, int lane, float (&z)[E]) {
  const T* p = static_cast<const T*>(a.logits) + (long long)t * a.ld + lane * E;
  if (VEC) {  // 16 bytes of fp32 or 8 of bf16 at a time, K a multiple of four
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const bool ok = in && lane * E + i < a.K;
      if (sizeof(T) == 4) {
        float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (ok) v = *reinterpret_cast<const float4*>(p + i);
        z[i] = v.x; z[i + 1] = v.y; z[i + 2] = v.z; z[i + 3] = v.w;
      } else {
        uint2 v = make_uint2(0xff80ff80u, 0xff80ff80u);  // -inf
        if (ok) v = *reinterpret_cast<const uint2*>(p + i);
        z[i] = __uint_as_float(v.x << 16);
        z[i + 1] = __uint_as_float(v.x & 0xffff0000u);
        z[i + 2] = __uint_as_float(v.y << 16);
        z[i + 3] = __uint_as_float(v.y & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) z[i] = in && lane * E + i < a.K ? to_float(p[i]) : -INFINITY;
  }
}

template <int E, bool VEC>
__device__ __forceinline__ void store(const Args& a, long long t, int lane, const float (&v)[E]) {
  float* to = a.dlogits + t * a.K + lane * E;
#pragma unroll
  for (int i = 0; i < E; i += 4) {
    if (VEC) {
      if (lane * E + i < a.K)
        *reinterpret_cast<float4*>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
      for (int k = i; k < i + 4; ++k)
        if (lane * E + k < a.K) to[k] = v[k];
    }
  }
}

// z to exp(z - max) (0 past K), their sum and the maximum; false for padding and for
// a token whose logits are all -inf.
template <int L, int E>
__device__ __forceinline__ bool softmax(bool in, float (&z)[E], float& top, float& sum) {
  top = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) top = fmaxf(top, z[i]);
  top = lanes_max<L>(top);
  const float base = top == -INFINITY ? 0.f : top;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    z[i] = __expf(z[i] - base);
    sum += z[i];
  }
  sum = lanes_sum<L>(sum);
  return in && (top != -INFINITY || isnan(sum));
}

// TH threads; U tokens of each group of lanes are loaded before the first is used.
template <typename T, int L, int E, bool VEC, int TH, int U>
__global__ void __launch_bounds__(TH) sums_kernel(const Args a) {
  constexpr int kWarps = TH / 32;
  extern __shared__ float sh[];  // [kWarps][K] probabilities, then [K] counts
  __shared__ float z_sh[kWarps];
  __shared__ int n_sh[kWarps];
  int* cnt = reinterpret_cast<int*>(sh + kWarps * a.K);
  for (int i = threadIdx.x; i < a.K; i += TH) cnt[i] = 0;
  __syncthreads();
  constexpr int kTok = TH / L;  // tokens of a CTA at a time
  const int lane = threadIdx.x % L, tok = threadIdx.x / L, warp = threadIdx.x / 32;
  const long long stride = (long long)gridDim.x * kTok;
  float p[E], zs = 0.f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) p[i] = 0.f;
  for (long long base = (long long)blockIdx.x * kTok; base < a.T; base += U * stride) {
    float z[U][E];
    int m[U], q0[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long tt = base + u * stride + tok;
      in[u] = tt < a.T && (!a.mask || a.mask[tt]);
      const int t = in[u] ? (int)tt : 0;
      load<T, L, E, VEC>(a, in[u], t, lane, z[u]);
      m[u] = a.n_q;
      q0[u] = -1;
      if (in[u]) {
        if (a.k) m[u] = min(m[u], a.k[t]);
        if (lane < a.n_q) q0[u] = a.q[(long long)t * a.ld_q + lane];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float top, sum;
      if (softmax<L, E>(in[u], z[u], top, sum)) {
        const float inv = 1.f / sum, lse = top + logf(sum);
#pragma unroll
        for (int i = 0; i < E; ++i) p[i] = fmaf(z[u][i], inv, p[i]);
        if (lane == 0) {
          zs = fmaf(lse, lse, zs);
          ++n;
        }
        int j = q0[u];
        for (int i = lane; i < m[u]; i += L) {
          if (i != lane) j = a.q[(base + u * stride + tok) * a.ld_q + i];
          if (j >= 0 && j < a.K) atomicAdd(&cnt[j], 1);
        }
      }
    }
  }
  // the groups of a warp, then the warps, in a fixed order
#pragma unroll
  for (int i = 0; i < E; ++i) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) p[i] += __shfl_xor_sync(0xffffffffu, p[i], o);
    const int c = lane * E + i;
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
  for (int c = threadIdx.x; c < a.K; c += TH) {
    float s = 0.f;
#pragma unroll 8
    for (int w = 0; w < kWarps; ++w) s += sh[w * a.K + c];
    a.part_p[(long long)c * gridDim.x + blockIdx.x] = s;
    a.part_c[(long long)c * gridDim.x + blockIdx.x] = cnt[c];
  }
  if (warp == kWarps - 1) {
    const int l = threadIdx.x & 31;
    float s = l < kWarps ? z_sh[l] : 0.f;
    int m = l < kWarps ? n_sh[l] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      m += __shfl_xor_sync(0xffffffffu, m, o);
    }
    if (l == 0) {
      a.part_z[blockIdx.x] = s;
      a.part_n[blockIdx.x] = m;
    }
  }
}

template <typename T, int L, int E, bool VEC, int TH, int U>
__global__ void __launch_bounds__(TH) gradient_kernel(const Args a) {
  constexpr int kWarps = TH / 32;
  extern __shared__ float f[];  // [K] f, then [K] mean probabilities (first CTA)
  __shared__ Total all_c;  // selections of all tokens
  __shared__ int all_n;
  __shared__ float zsum;
  float* prob = f + a.K;
  const int lane32 = threadIdx.x & 31, warp = threadIdx.x / 32;
  const bool first = blockIdx.x == 0;
  if (threadIdx.x == 0) all_c.clear();
  grid_dep_wait();
  __syncthreads();
  // a warp per column adds the CTAs' sums (whole numbers, and in a fixed order)
  for (int c = warp; c < a.K; c += kWarps) {
    long long m = 0;
    float q = 0.f;
    for (int i = lane32; i < a.ctas; i += 32) {
      m += a.part_c[(long long)c * a.ctas + i];
      if (first) q += a.part_p[(long long)c * a.ctas + i];
    }
    m = warp_total(m);
    q = lanes_sum<32>(q);
    if (lane32 == 0) {
      f[c] = (float)m;
      all_c.add(m);
      if (first) {
        prob[c] = q;
        a.counts[c] = count32(m);
      }
    }
  }
  if (warp == kWarps - 1) {
    int n = 0;
    float z = 0.f;
    for (int i = lane32; i < a.ctas; i += 32) {
      n += a.part_n[i];
      if (first) z += a.part_z[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      n += __shfl_xor_sync(0xffffffffu, n, o);
      z += __shfl_xor_sync(0xffffffffu, z, o);
    }
    if (lane32 == 0) {
      all_n = n;
      zsum = z;
    }
  }
  __syncthreads();
  const float inv_c = 1.f / (float)max(all_c.get(), 1ll), inv_n = 1.f / (float)max(all_n, 1);
  for (int c = threadIdx.x; c < a.K; c += TH) f[c] *= inv_c;
  __syncthreads();
  if (first && warp == 0) {
    float b = 0.f;
    for (int c = lane32; c < a.K; c += 32) {
      const float q = prob[c] * inv_n;
      a.prob[c] = q;
      b = fmaf(f[c], q, b);
    }
    b = lanes_sum<32>(b) * (float)a.K;
    if (lane32 == 0) {
      const float z = zsum * inv_n;
      a.loss[0] = fmaf(a.w_b, b, a.w_z * z);
      a.loss[1] = b;
      a.loss[2] = z;
    }
  }
  if (!a.dlogits) return;
  constexpr int kTok = TH / L;
  const int lane = threadIdx.x % L, tok = threadIdx.x / L;
  const float wb = a.w_b * (float)a.K, wz = 2.f * a.w_z;
  const long long stride = (long long)gridDim.x * kTok;
  float fr[E];
#pragma unroll
  for (int i = 0; i < E; ++i) fr[i] = lane * E + i < a.K ? f[lane * E + i] : 0.f;
  for (long long base = (long long)blockIdx.x * kTok; base < a.T; base += U * stride) {
    float e[U][E];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long tt = base + u * stride + tok;
      in[u] = tt < a.T && (!a.mask || a.mask[tt]);
      load<T, L, E, VEC>(a, in[u], in[u] ? (int)tt : 0, lane, e[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long tt = base + u * stride + tok;
      float top, sum;
      const bool valid = softmax<L, E>(in[u], e[u], top, sum);
      const float inv = 1.f / sum;
      float fp = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        e[u][i] *= inv;
        fp = fmaf(fr[i], e[u][i], fp);
      }
      fp = lanes_sum<L>(fp);
      const float g = fmaf(wz, top + logf(sum), -wb * fp);
#pragma unroll
      for (int i = 0; i < E; ++i) e[u][i] = valid ? e[u][i] * inv_n * fmaf(wb, fr[i], g) : 0.f;
      if (tt < a.T) store<E, VEC>(a, tt, lane, e[u]);
    }
  }
}

__device__ __forceinline__ uint32_t of_rank(const void* p, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t read_rank(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                   : "memory");
}

// The whole call in one kernel, where a cluster of CTAs holds all tokens'
// probabilities in its registers (up to U tokens per group of lanes): the CTAs
// read one another's column sums from shared memory. Two kernels cost a second
// launch and a second reading.
template <typename T, int L, int E, bool VEC, int TH, int U>
__global__ void __launch_bounds__(TH) cluster_kernel(const Args a) {
  constexpr int kWarps = TH / 32, kTok = TH / L;
  extern __shared__ float sh[];  // [kWarps][K] shares; then [K] sums, [K] counts, [K] f
  __shared__ float z_sh[kWarps], zsum;
  __shared__ int n_sh[kWarps], all_n, mine[2];
  __shared__ Total all_c;
  float* sum_p = sh + kWarps * a.K;
  int* cnt = reinterpret_cast<int*>(sum_p + a.K);
  float* f = sum_p + 2 * a.K;
  const int lane = threadIdx.x % L, tok = threadIdx.x / L, warp = threadIdx.x / 32,
            lane32 = threadIdx.x & 31;
  const uint32_t ranks = gridDim.x;  // one cluster
  const int held = (int)((a.T + ranks * kTok - 1) / (ranks * kTok));  // tokens of a group, <= U
  for (int i = threadIdx.x; i < a.K; i += TH) cnt[i] = 0;
  if (threadIdx.x == 0) all_c.clear();
  float z[U][E], lse[U];
  int m[U], q0[U];
  bool in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= held) break;
    const int t0 = (u * (int)ranks + (int)blockIdx.x) * kTok + tok;
    in[u] = t0 < a.T && (!a.mask || a.mask[t0]);
    const int t = in[u] ? t0 : 0;
    load<T, L, E, VEC>(a, in[u], t, lane, z[u]);
    m[u] = a.n_q;
    q0[u] = -1;
    if (in[u]) {
      if (a.k) m[u] = min(m[u], a.k[t]);
      if (lane < a.n_q) q0[u] = a.q[(long long)t * a.ld_q + lane];
    }
  }
  __syncthreads();
  float p[E], zs = 0.f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) p[i] = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= held) break;
    float top, sum;
    in[u] = softmax<L, E>(in[u], z[u], top, sum);
    const float inv = 1.f / sum;
    lse[u] = top + logf(sum);
#pragma unroll
    for (int i = 0; i < E; ++i) z[u][i] *= inv;
    if (in[u]) {
#pragma unroll
      for (int i = 0; i < E; ++i) p[i] += z[u][i];
      if (lane == 0) {
        zs = fmaf(lse[u], lse[u], zs);
        ++n;
      }
      const long long t = (u * (int)ranks + (int)blockIdx.x) * kTok + tok;
      int j = q0[u];
      for (int i = lane; i < m[u]; i += L) {
        if (i != lane) j = a.q[t * a.ld_q + i];
        if (j >= 0 && j < a.K) atomicAdd(&cnt[j], 1);
      }
    }
  }
  // the groups of a warp, the warps, then the CTAs, in a fixed order
#pragma unroll
  for (int i = 0; i < E; ++i) {
#pragma unroll
    for (int o = L; o < 32; o <<= 1) p[i] += __shfl_xor_sync(0xffffffffu, p[i], o);
    const int c = lane * E + i;
    if (lane32 < L && c < a.K) sh[warp * a.K + c] = p[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    zs += __shfl_xor_sync(0xffffffffu, zs, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if (lane32 == 0) {
    z_sh[warp] = zs;
    n_sh[warp] = n;
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.K; c += TH) {
    float s = 0.f;
#pragma unroll 8
    for (int w = 0; w < kWarps; ++w) s += sh[w * a.K + c];
    sum_p[c] = s;
  }
  if (warp == kWarps - 1) {
    float s = lane32 < kWarps ? z_sh[lane32] : 0.f;
    int k = lane32 < kWarps ? n_sh[lane32] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      k += __shfl_xor_sync(0xffffffffu, k, o);
    }
    if (lane32 == 0) {
      mine[0] = __float_as_int(s);
      mine[1] = k;
    }
  }
  cluster_sync();
  const bool first = blockIdx.x == 0;
  long long total = 0;
  for (int c = threadIdx.x; c < a.K; c += TH) {
    long long k = 0;
    float s = 0.f;
    for (uint32_t r = 0; r < ranks; ++r) {
      k += (int)read_rank(of_rank(cnt + c, r));
      if (first) s += __uint_as_float(read_rank(of_rank(sum_p + c, r)));
    }
    f[c] = (float)k;
    total += k;
    if (first) {
      a.counts[c] = count32(k);
      sh[c] = s;  // (the shares have been added)
    }
  }
  total = warp_total(total);
  if (lane32 == 0) all_c.add(total);
  if (threadIdx.x == TH - 1) {
    int k = 0;
    float s = 0.f;
    for (uint32_t r = 0; r < ranks; ++r) {
      s += __uint_as_float(read_rank(of_rank(&mine[0], r)));
      k += (int)read_rank(of_rank(&mine[1], r));
    }
    zsum = s;
    all_n = k;
  }
  cluster_sync();  // nothing is read from another CTA any more; all of this CTA's is written
  const float inv_c = 1.f / (float)max(all_c.get(), 1ll), inv_n = 1.f / (float)max(all_n, 1);
  if (first && warp == 0) {
    float b = 0.f;
    for (int c = lane32; c < a.K; c += 32) {
      const float q = sh[c] * inv_n;
      a.prob[c] = q;
      b = fmaf(f[c] * inv_c, q, b);
    }
    b = lanes_sum<32>(b) * (float)a.K;
    if (lane32 == 0) {
      const float zl = zsum * inv_n;
      a.loss[0] = fmaf(a.w_b, b, a.w_z * zl);
      a.loss[1] = b;
      a.loss[2] = zl;
    }
  }
  if (!a.dlogits) return;
  const float wb = a.w_b * (float)a.K, wz = 2.f * a.w_z;
  float fr[E];
#pragma unroll
  for (int i = 0; i < E; ++i)
    fr[i] = lane * E + i < a.K ? f[lane * E + i] * inv_c : 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= held) break;
    const int t = (u * (int)ranks + (int)blockIdx.x) * kTok + tok;
    float fp = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) fp = fmaf(fr[i], z[u][i], fp);
    fp = lanes_sum<L>(fp);
    const float g = fmaf(wz, lse[u], -wb * fp);
#pragma unroll
    for (int i = 0; i < E; ++i) z[u][i] = in[u] ? z[u][i] * inv_n * fmaf(wb, fr[i], g) : 0.f;
    if (t < a.T) store<E, VEC>(a, t, lane, z[u]);
  }
}

constexpr int kWide = 128;  // up to this many experts: CTAs of 1,024 threads
inline int threads_of(int K) { return K <= kWide ? 1024 : 256; }

// Whether clusters of 16 CTAs of this kernel can run on the current device (above the
// portable eight); lets them be launched there.
bool allow_cluster_16(const void* fn, int threads, size_t smem) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int clusters = 0;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
      cudaOccupancyMaxActiveClusters(&clusters, fn, &cfg) == cudaSuccess && clusters > 0)
    return true;
  cudaGetLastError();  // a refusal is no error of the call
  return false;
}

// The most CTAs of a cluster of this kernel on the current device: 16 where it takes that
// many (not every one has to), else 8.
unsigned largest_cluster(const void* fn, int threads, size_t smem) {
  static PerDevice<unsigned> kept;
  int dev = 0;
  unsigned n = 8;
  if (cudaGetDevice(&dev) != cudaSuccess) return n;
  try {
    kept.get(fn, dev, &n, [&](unsigned* to) {
      *to = allow_cluster_16(fn, threads, smem) ? 16 : 8;
      return true;
    });
  } catch (...) {  // no exception leaves the library
    return 8;
  }
  return n;
}

// Lanes per token, and tokens that a cluster of eight CTAs holds at once (those of
// cluster_kernel's instances).
int lanes_of(int K) {
  return K <= 4 ? 1 : K <= 8 ? 2 : K <= 16 ? 4 : K <= 32 ? 8 : K <= 64 ? 16 : 32;
}
bool in_cluster(int T, int K) {
  return T <= 8ll * (K <= 256 ? 4 : 2) * (threads_of(K) / lanes_of(K));
}

// CTAs of both kernels: at most one per SM, so that the second has few sums to add.
int cta_count(int T, int K, int sms) {
  const long long tok = threads_of(K) / lanes_of(K), want = ((long long)T + tok - 1) / tok;
  return (int)(want < 1 ? 1 : want > sms ? sms : want);
}

// The most tokens that one CTA takes. Its counts are 32-bit, the sums over CTAs are not.
long long tokens_per_cta(int T, int K, int ctas) {
  const long long tok = threads_of(K) / lanes_of(K);
  // (a cluster of eight: up to four tokens of each group of lanes)
  const long long most = in_cluster(T, K) ? 4 * tok : ((T + tok - 1) / tok + ctas - 1) / ctas * tok;
  return most < T ? most : T;
}

template <typename T, int L, int E, bool VEC, int TH, int U>
cudaError_t launch_as(const Args& a, cudaStream_t s) {
  if (in_cluster(a.T, a.K)) {
    // as many CTAs as have tokens, up to the largest cluster
    const unsigned most = largest_cluster(
        reinterpret_cast<const void*>(cluster_kernel<T, L, E, VEC, TH, U>), TH,
        (size_t)(TH / 32 + 3) * a.K * sizeof(float));
    unsigned ctas = 1;
    while (ctas < most && (long long)ctas * (TH / L) < a.T) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(TH);
    cfg.dynamicSmemBytes = (size_t)(TH / 32 + 3) * a.K * sizeof(float);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cluster_kernel<T, L, E, VEC, TH, U>, a);
  }
  const size_t smem = (size_t)(TH / 32 * a.K + a.K) * sizeof(float);
  const size_t smem2 = (size_t)(2 * a.K) * sizeof(float);
  sums_kernel<T, L, E, VEC, TH, U><<<a.ctas, TH, smem, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_dependent(gradient_kernel<T, L, E, VEC, TH, U>, dim3(a.dlogits ? a.ctas : 1), dim3(TH),
                          smem2, s, a);
}

template <typename T, bool VEC>
cudaError_t launch(const Args& a, cudaStream_t s) {
  if (a.K <= 4) return launch_as<T, 1, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 8) return launch_as<T, 2, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 16) return launch_as<T, 4, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 32) return launch_as<T, 8, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 64) return launch_as<T, 16, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 128) return launch_as<T, 32, 4, VEC, 1024, 4>(a, s);
  if (a.K <= 256) return launch_as<T, 32, 8, VEC, 256, 4>(a, s);
  return launch_as<T, 32, 16, VEC, 256, 2>(a, s);
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
  return bl::in_cluster(T, K) ? 0 : bl::layout(K, bl::cta_count(T, K, sms), at);
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
  int sms = 1;
  if (!bl::in_cluster(T, K)) {
    const int rs = unif::sm_count(&sms);
    if (rs != UNIF_MOE_OK) return rs;
  }
  bl::Args a{};
  a.ctas = bl::cta_count(T, K, sms);
  if (bl::tokens_per_cta(T, K, a.ctas) * n_q > 0x7fff0000) {  // (a lane's index goes 32 beyond)
    set_error("n_q=%d: too many selections for one CTA's tokens", n_q);
    return UNIF_MOE_ERR_SHAPE;
  }
  int64_t at[4] = {};
  const int64_t need = bl::in_cluster(T, K) ? 0 : bl::layout(K, a.ctas, at);
  if (workspace_bytes < need || (need && !workspace)) {
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
  const uintptr_t step = dtype == UNIF_MOE_BF16 ? 8 : 16;
  const bool vec = K % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(logits) % step == 0 &&
                   reinterpret_cast<uintptr_t>(dlogits) % 16 == 0;
  cudaError_t e;
  if (dtype == UNIF_MOE_BF16)
    e = vec ? bl::launch<__nv_bfloat16, true>(a, s) : bl::launch<__nv_bfloat16, false>(a, s);
  else
    e = vec ? bl::launch<float, true>(a, s) : bl::launch<float, false>(a, s);
  if (e != cudaSuccess) {
    set_error("balance loss: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

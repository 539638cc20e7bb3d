// The norms round a block, fused with the block's gate and the scaled residual
// sum, forward and backward (unif_moe_block_norm_forward / _backward).
//
//   yn = (y - mean) rstd,  z = w_post yn + b_post      (or z = y)
//   out = s x + g z,  u = w_pre (out - mean) rstd + b_pre
//
// Both passes are bound by memory: a row is read once, held in registers while
// its sums are taken, and its results written once. A row belongs to a group of
// threads, eight values to a thread: 8, 16 or 32 lanes of a warp where d <= 64,
// 128 or 256, else a CTA of ceil(d / 256) warps. Values and sums are fp32; a result is
// rounded once, to the type it is stored in.
//
// Measured (us; at the copy rate of 6.8 TB/s): forward of 12,608 x 384, fp32 stream,
// 12.9 (8.6), of 20,000 x 1,024 bf16 with norms on both sides 38 (24); backward of 12,608 x 768
// bf16 with a gate per image 34 (17), of 65,536 x 1,024 padded, fp32 stream, 189 (126
// for the rows that are read, 178 for all). Widths that are no multiple of eight move value by value: backward
// of 20,000 x 1,001 bf16 104 (35), forward 67 (24).
#include <cuda_bf16.h>
#include <math.h>

#include "internal.cuh"

namespace unif {
namespace norm {

constexpr int kE = 8;            // values per thread and row
constexpr int kThreads = 128;    // threads per CTA of the forms with several rows per warp or CTA
constexpr int kMaxWarps = 32;

// ---- eight values of a row ----
// VEC: thread j of a group holds columns 8 j .. 8 j + 7 (one access of 16 bytes of bf16
// or 32 of fp32: whole sectors); otherwise columns j, j + n, j + 2 n, ... of n threads.
template <bool VEC>
__device__ __forceinline__ int column(int j, int n, int i) {
  return VEC ? j * kE + i : i * n + j;
}

__device__ __forceinline__ void unpack(const uint4& r, float (&v)[kE]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

template <bool VEC>
__device__ __forceinline__ void load(const float* p, int j, int n, int d, float (&v)[kE]) {
  if (VEC) {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = 0.f;
    if (j * kE < d)
      asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]),
                     "=f"(v[6]), "=f"(v[7])
                   : "l"(p + j * kE)
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      v[i] = 0.f;
      if (i * n < d && column<false>(j, n, i) < d) v[i] = p[column<false>(j, n, i)];
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void load(const __nv_bfloat16* p, int j, int n, int d, float (&v)[kE]) {
  if (VEC) {
    uint4 a = make_uint4(0u, 0u, 0u, 0u);
    if (j * kE < d) a = *reinterpret_cast<const uint4*>(p + j * kE);
    unpack(a, v);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      v[i] = 0.f;
      if (i * n < d && column<false>(j, n, i) < d) v[i] = __bfloat162float(p[column<false>(j, n, i)]);
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void store(float* p, int j, int n, int d, const float (&v)[kE]) {
  if (VEC) {
    if (j * kE < d)
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + j * kE),
                   "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]),
                   "f"(v[7])
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i * n < d && column<false>(j, n, i) < d) p[column<false>(j, n, i)] = v[i];
  }
}
template <bool VEC>
__device__ __forceinline__ void store(__nv_bfloat16* p, int j, int n, int d, const float (&v)[kE]) {
  if (VEC) {
    if (j * kE < d) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t*>(&t);
      }
      *reinterpret_cast<uint4*>(p + j * kE) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i * n < d && column<false>(j, n, i) < d) p[column<false>(j, n, i)] = __float2bfloat16_rn(v[i]);
  }
}

// The sums of N values over the threads of a row's group. GL: lanes per group
// within a warp, or 0 for the whole CTA; the warps of a CTA meet in `red` (two
// buffers in turn: the next sum writes the other one, so one barrier is enough).
template <int GL, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* red, int& turn) {
#pragma unroll
  for (int o = (GL ? GL : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (GL) return;
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  float* buf = red + (turn & 1) * (2 * kMaxWarps);
  turn ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) buf[(threadIdx.x >> 5) * N + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += buf[w * N + i];
}

// ---- forward ----
template <typename TX, typename TB>
struct ForwardArgs {
  int T, d, post, pre, gate_rows;
  float scale, eps;
  const TX* x;
  const TB* y;
  long long ld_x, ld_y, ld_out, ld_u;
  const uint8_t* mask;
  const TB *w_post, *b_post, *gate, *w_pre, *b_pre;
  TX* out;
  TB* u;
  float *m_post, *r_post, *m_pre, *r_pre;
};

// One row to a group of threads. MT: most threads of a CTA; without VEC the threads, so
// that the columns' offsets are constants (with an offset and a bound worked out per
// value, a row of 333 took 1,850 instructions a warp in the backward). With VEC a thread keeps
// to 32 registers (else 40), so that all 64 warps are on an SM (9,728 x 4,096 fp32 124 us with one CTA, 98
// with two; bf16 parameters 8,192 wide 218 and 208). Not in groups of fp32 vectors, which would
// spill (155,648 x 64 27.1 us, 28.2 so).
template <typename TB, bool VEC, int GL, int MT>
constexpr int least_ctas() {
  return !VEC ? 1536 / MT : GL && sizeof(TB) == 4 ? 1 : 2048 / MT;
}
template <typename TX, typename TB, bool VEC, int GL, int MT>
__global__ void __launch_bounds__(MT, least_ctas<TB, VEC, GL, MT>())
    forward_kernel(const ForwardArgs<TX, TB> a) {
  __shared__ float red[2 * 2 * kMaxWarps];
  int turn = 0;
  const int n = GL ? GL : VEC ? (int)blockDim.x : MT;
  const int j = GL ? (int)threadIdx.x % (GL ? GL : 1) : (int)threadIdx.x;
  const int rows = GL ? kThreads / (GL ? GL : 1) : 1;
  const int d = a.d;
  // every lane of a warp takes part in the shuffles, also past the last row
  const int row = blockIdx.x * rows + (GL ? (int)threadIdx.x / (GL ? GL : 1) : 0);
  const bool in = row < a.T, valid = in && (!a.mask || a.mask[row]);
  const bool act = valid && (!VEC || j * kE < d);  // has columns of a row that counts
  float o[kE], z[kE];
#pragma unroll
  for (int i = 0; i < kE; ++i) o[i] = z[i] = 0.f;
  if (act) {
    load<VEC>(a.x + row * a.ld_x, j, n, d, o);
    if (a.y) load<VEC>(a.y + row * a.ld_y, j, n, d, z);
  }
  float mean = 0.f, rstd = 0.f;
  const float inv = 1.f / (float)d;
  auto norm = [&](float (&v)[kE], int kind, const TB* w, const TB* b) {
    if (!GL && !valid) return;  // (the whole CTA)
    float s[1] = {0.f}, t[kE];
    mean = 0.f;
    if (kind == UNIF_MOE_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < kE; ++i) s[0] += v[i];
      group_sum<GL>(s, red, turn);
      mean = s[0] * inv;
      const float m = act ? mean : 0.f;  // columns past d hold 0 and stay 0
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (VEC || column<false>(j, n, i) < d) v[i] -= m;
      s[0] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) s[0] = fmaf(v[i], v[i], s[0]);
    group_sum<GL>(s, red, turn);
    rstd = rsqrtf(s[0] * inv + a.eps);
    if (!act) return;
    load<VEC>(w, j, n, d, t);
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = v[i] * rstd * t[i];
    if (b) {
      load<VEC>(b, j, n, d, t);
#pragma unroll
      for (int i = 0; i < kE; ++i) v[i] += t[i];
    }
  };
  if (a.y) {
    if (a.post) {
      norm(z, a.post, a.w_post, a.b_post);
      if (j == 0 && in) {
        if (a.m_post) a.m_post[row] = valid ? mean : 0.f;
        if (a.r_post) a.r_post[row] = valid ? rstd : 0.f;
      }
    }
    if (act) {
      if (a.gate) {
        float g[kE];
        load<VEC>(a.gate_rows ? a.gate + (long long)(row / a.gate_rows) * d : a.gate, j, n, d, g);
#pragma unroll
        for (int i = 0; i < kE; ++i) z[i] *= g[i];
      }
#pragma unroll
      for (int i = 0; i < kE; ++i) o[i] = fmaf(a.scale, o[i], z[i]);
    }
    if (a.out && in) store<VEC>(a.out + row * a.ld_out, j, n, d, o);
  }
  if (a.pre) {
    norm(o, a.pre, a.w_pre, a.b_pre);
    if (in) {
      store<VEC>(a.u + row * a.ld_u, j, n, d, o);
      if (j == 0) {
        if (a.m_pre) a.m_pre[row] = valid ? mean : 0.f;
        if (a.r_pre) a.r_pre[row] = valid ? rstd : 0.f;
      }
    }
  }
}

// ---- pairs of fp32 values (one instruction for two) ----
struct F8 {
  uint64_t p[kE / 2];
};
__device__ __forceinline__ uint64_t pk(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 upk(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ F8 pairs(const float (&v)[kE]) {
  F8 r;
#pragma unroll
  for (int i = 0; i < kE / 2; ++i) r.p[i] = pk(v[2 * i], v[2 * i + 1]);
  return r;
}
__device__ __forceinline__ void singles(const F8& a, float (&v)[kE]) {
#pragma unroll
  for (int i = 0; i < kE / 2; ++i) {
    const float2 f = upk(a.p[i]);
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ F8 zero8() {
  F8 r;
#pragma unroll
  for (int i = 0; i < kE / 2; ++i) r.p[i] = 0ull;
  return r;
}

// Sums over the threads of a row's group of two values for each of R rows, each
// given as a pair of partial sums. N = 2 R values are halved among the lanes at
// every exchange until a lane carries one: N - 1 + log2(lanes / N) shuffles. The
// warps of a CTA meet in `red` (two buffers in turn), of which they read all
// `W` warps' slots, those without a warp being 0.
template <int GL, int R, int W>
__device__ __forceinline__ void group_sums(const uint64_t (&s)[R][2], float* red, int& turn,
                                           float2 (&out)[R]) {
  constexpr int N = 2 * R, kLanes = GL ? GL : 32;
  float v[N];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float2 a = upk(s[r][0]), b = upk(s[r][1]);
    v[2 * r] = a.x + a.y;
    v[2 * r + 1] = b.x + b.y;
  }
  // after the exchanges lane l carries value (l / (kLanes / N)) of its group
  int half = kLanes / 2;
#pragma unroll
  for (int m = N / 2; m > 0; m >>= 1, half >>= 1) {
    const bool upper = threadIdx.x & half;
#pragma unroll
    for (int i = 0; i < m; ++i)
      v[i] = (upper ? v[m + i] : v[i]) + __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[m + i], half);
  }
#pragma unroll
  for (; half > 0; half >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], half);
  constexpr int kStep = kLanes / N;
  if (GL) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int at = (threadIdx.x & 31 & ~(kLanes - 1)) + 2 * r * kStep;
      out[r].x = __shfl_sync(0xffffffffu, v[0], at);
      out[r].y = __shfl_sync(0xffffffffu, v[0], at + kStep);
    }
    return;
  }
  float* buf = red + (turn & 1) * (N * W);
  turn ^= 1;
  if ((threadIdx.x & (kStep - 1)) == 0) buf[threadIdx.x / kStep] = v[0];  // warp w: N w ...
  __syncthreads();
  uint64_t t[R];
#pragma unroll
  for (int r = 0; r < R; ++r) t[r] = reinterpret_cast<const uint64_t*>(buf)[r];
#pragma unroll
  for (int w = 1; w < W; ++w)
#pragma unroll
    for (int r = 0; r < R; ++r) t[r] = add2(t[r], reinterpret_cast<const uint64_t*>(buf)[w * R + r]);
#pragma unroll
  for (int r = 0; r < R; ++r) out[r] = upk(t[r]);
}

// Eight values of a row that is not moved 16 bytes at a time: on their way (Coming: no
// instruction uses them yet, so nothing waits for them) and held.
template <typename T>
struct Coming {
  T v[kE];
  __device__ __forceinline__ void read(const T* p, int j, int n, int d) {
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      v[i] = (T)0;
      if (i * n < d && column<false>(j, n, i) < d) v[i] = p[column<false>(j, n, i)];
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = (T)0;
  }
};
template <typename T>
struct Bits {  // what a value is read as
  using type = float;
};
template <>
struct Bits<__nv_bfloat16> {
  using type = unsigned short;
};
template <typename T>
struct Row8;
template <>
struct Row8<float> {
  float v[kE];
  __device__ __forceinline__ void take(const Coming<float>& c) {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = c.v[i];
  }
  __device__ __forceinline__ F8 get() const { return pairs(v); }
};
template <>
struct Row8<__nv_bfloat16> {
  uint4 raw;
  __device__ __forceinline__ void take(const Coming<unsigned short>& c) {
    uint32_t h[kE / 2];
#pragma unroll
    for (int i = 0; i < kE / 2; ++i) h[i] = (uint32_t)c.v[2 * i] | (uint32_t)c.v[2 * i + 1] << 16;
    raw = make_uint4(h[0], h[1], h[2], h[3]);
  }
  __device__ __forceinline__ void read(const __nv_bfloat16* p, int j, int n, int d) {
    Coming<unsigned short> c;
    c.read(reinterpret_cast<const unsigned short*>(p), j, n, d);
    take(c);
  }
  __device__ __forceinline__ void clear() { raw = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ F8 get() const {
    float v[kE];
    unpack(raw, v);
    return pairs(v);
  }
};

// A parameter's values of this thread's columns (0 where it is NULL or not `on`): bf16 ones
// stay in registers from row to row as they were read, fp32 ones are read again.
template <typename TB, bool VEC>
struct Param {
  const TB* p = nullptr;
  __device__ __forceinline__ void set(const TB* q, int, int, int) { p = q; }
  __device__ __forceinline__ F8 get(int j, int n, int d, bool on = true) const {
    if (!p || !on) return zero8();
    float v[kE];
    load<VEC>(p, j, n, d, v);
    return pairs(v);
  }
};
template <>
struct Param<__nv_bfloat16, false> {
  Row8<__nv_bfloat16> held;
  __device__ __forceinline__ Param() { held.clear(); }
  __device__ __forceinline__ void set(const __nv_bfloat16* q, int j, int n, int d) {
    held.clear();
    if (q) held.read(q, j, n, d);
  }
  __device__ __forceinline__ F8 get(int, int, int, bool on = true) const {
    return on ? held.get() : zero8();
  }
};
template <>
struct Param<__nv_bfloat16, true> {
  uint4 raw = {0u, 0u, 0u, 0u};
  __device__ __forceinline__ void set(const __nv_bfloat16* q, int j, int, int d) {
    raw = make_uint4(0u, 0u, 0u, 0u);
    if (q && j * kE < d) raw = *reinterpret_cast<const uint4*>(q + j * kE);
  }
  __device__ __forceinline__ F8 get(int, int, int, bool on = true) const {
    float v[kE];
    unpack(on ? raw : make_uint4(0u, 0u, 0u, 0u), v);
    return pairs(v);
  }
};

// ---- backward ----
// With o^ = (out - m) r, a = du w_pre:
//   D = dout + r (a - mean(a) - o^ mean(a o^)),  dx = s D
//   e = D g,  f = e w_post,  dy = r_y (f - mean(f) - yn mean(f yn))
// (no mean(a), mean(f) terms for rms), and the column sums
//   dw_pre = sum du o^, db_pre = sum du, dw_post = sum e yn, db_post = sum e,
//   dg = sum D z over the rows of a gate row.
// A CTA walks rows that share a gate row, every pieces-th chunk of them so that
// padding falls on all CTAs alike, or a run of whole gate rows. It keeps the column sums of its columns in registers and writes
// them once; finish_kernel adds the CTAs' sums in a fixed order, so results
// do not change from run to run.
template <typename TX, typename TB>
struct BackwardArgs {
  int T, d, post, pre, gate_rows;
  float scale;
  const TX* o;
  const TB* y;
  const TX* dout;
  const TB* du;
  long long ld_o, ld_y, ld_dout, ld_du, ld_dx, ld_dy;
  const uint8_t* mask;
  const TB *w_post, *b_post, *gate, *w_pre;
  const float *m_post, *r_post, *m_pre, *r_pre;
  TX* dx;
  TB* dy;
  float* d_gate;       // written here where a CTA holds whole gate rows (pieces == 1)
  float* part;         // [CTAs][4][d]: dw_post, db_post, dw_pre, db_pre
  float* part_gate;    // [CTAs][d] where pieces > 1
  int wanted;          // bits 0-3: the sums of part; bit 4: dg
  int pieces;          // CTAs per gate row, or 1
  int run;             // rows per CTA (pieces == 1), or of a chunk
};

// A step of the backward takes R rows of a group at a time (two, where the threads
// are few enough to have the registers); the next steps' rows are on their way to
// shared memory meanwhile, in a ring of as many steps as the SM's shared memory
// holds for 384 or 512 threads.
__host__ __device__ constexpr int step_rows(bool vec, int mt) { return vec && mt <= 384 ? 2 : 1; }
template <typename TX, typename TB>
__host__ __device__ constexpr int row_bytes() {  // of a thread: dout, out, y, du
  return 2 * kE * (int)(sizeof(TX) + sizeof(TB));
}
template <typename TX, typename TB>
__host__ __device__ constexpr int ring_steps(int mt) {
  return (mt <= 384 ? 512 : 384) / (step_rows(true, mt) * row_bytes<TX, TB>());
}

// This thread's eight values of a row, global to shared (16-byte planes of
// `threads` slots each) and back: a thread reads only what it copied itself, so
// waiting for its own copies is enough.
template <typename T>
__device__ __forceinline__ void ring_copy(uint4* slot, const T* p, int threads) {
  constexpr int n = kE * sizeof(T) / 16;
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(slot + i * threads));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst),
                 "l"(reinterpret_cast<const uint4*>(p) + i)
                 : "memory");
  }
}
__device__ __forceinline__ void ring_read(const uint4* slot, int threads, const float*, float (&v)[kE]) {
  const uint4 a = slot[0], b = slot[threads];
  v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y);
  v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y);
  v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
}
__device__ __forceinline__ void ring_read(const uint4* slot, int, const __nv_bfloat16*, float (&v)[kE]) {
  unpack(slot[0], v);
}

// The rows of a CTA, `step` at a time: chunks of consecutive rows `skip` rows apart,
// or, with `cut`, one gate row after another (`gate` is the one it is in).
struct Walk {
  int base, end, last, size, skip, gate;
  bool cut;
  __device__ __forceinline__ bool more() const { return base < last; }
  __device__ __forceinline__ void next(int step) {
    base += step;
    if (base >= end) {
      base = last - end > skip ? end + skip : last;
      end = min(last - base, size) + base;
      if (cut) ++gate;
    }
  }
};

// MT: most threads of a CTA. Two rows at a time take about 160 registers, so 12
// warps are on an SM; with one row and 16 warps the chains of a row (two sums over
// the CTA) left half of the issue slots empty.
template <typename TX, typename TB, bool VEC, int GL, int MT>
__global__ void __launch_bounds__(MT, MT <= 384 ? 384 / MT : 1)
    backward_kernel(const BackwardArgs<TX, TB> a) {
  constexpr int R = step_rows(VEC, MT), W = MT / 32;
  constexpr int kRing = VEC ? ring_steps<TX, TB>(MT) : 2;
  // without VEC the next row waits in registers, where there are enough
  constexpr bool kHeld = !VEC && MT <= 512, kAhead = VEC || kHeld;
  constexpr int kPX = kE * sizeof(TX) / 16, kPB = kE * sizeof(TB) / 16;  // planes of an array
  constexpr int kPlanes = 2 * kPX + 2 * kPB;
  constexpr int kGroups = GL ? MT / (GL ? GL : 1) : 1;
  constexpr int kStep = kGroups * R;
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float red[GL ? 4 : 2 * 2 * R * W];
  __shared__ float fold[GL ? MT * kE : 1];
  const int threads = (int)blockDim.x;
  int turn = 0;
  const int n = GL ? GL : VEC ? threads : MT;
  const int j = GL ? (int)threadIdx.x % (GL ? GL : 1) : (int)threadIdx.x;
  const int grp = GL ? (int)threadIdx.x / (GL ? GL : 1) : 0;
  const int d = a.d;
  const float inv = 1.f / (float)d;
  const bool layer_pre = a.pre == UNIF_MOE_NORM_LAYER, layer_post = a.post == UNIF_MOE_NORM_LAYER;
  const bool act = !VEC || j * kE < d;  // VEC: this thread has columns
  const int period = a.gate_rows ? a.gate_rows : a.T;
  const bool sum_gate = (a.wanted & 16) != 0;
  const bool each = a.gate_rows == 1;  // a gate row for each row
  const bool cut = a.gate && a.pieces == 1 && !each;
  Walk at;
  at.cut = cut;
  if (a.pieces > 1) {  // every pieces-th chunk of a gate row
    at.gate = blockIdx.x / a.pieces;
    const int p = blockIdx.x % a.pieces, g0 = at.gate * period;
    at.last = min(a.T - g0, period) + g0;
    at.size = a.run;
    at.skip = (a.pieces - 1) * a.run;
    at.base = (int)min((long long)at.last, g0 + (long long)p * a.run);
  } else {
    at.base = (int)min((long long)a.T, (long long)blockIdx.x * a.run);
    at.last = min(a.T - at.base, a.run) + at.base;
    at.gate = at.base / period;
    at.size = cut ? period : a.run;
    at.skip = 0;
  }
  at.end = min(at.last - at.base, at.size) + at.base;
  const bool with_y = a.dy || (a.wanted & 19);
  F8 s_wpost = zero8(), s_bpost = zero8(), s_wpre = zero8(), s_bpre = zero8(), s_gate = zero8();

  // Adds the groups' sums of a column in order of the groups and stores them.
  auto flush = [&](F8& sum, float* to) {
    float s[kE];
    singles(sum, s);
    if (GL) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kE; ++i) fold[i * MT + threadIdx.x] = s[i];
      __syncthreads();
      if (grp == 0)
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          float t = 0.f;
          for (int g = 0; g < kGroups; ++g) t += fold[i * MT + g * n + j];
          s[i] = t;
        }
    }
    if (grp == 0) store<VEC>(to, j, n, d, s);
    sum = zero8();
  };
  Param<TB, VEC> w_pre, w_post, b_post, gate;
  w_pre.set(a.w_pre, j, n, d);
  w_post.set(a.w_post, j, n, d);
  b_post.set(a.b_post, j, n, d);
  if (a.gate && !each) gate.set(a.gate + (long long)at.gate * d, j, n, d);

  // planes of dout, out, y, du of each row of a step
  auto slot = [&](int k, int r) { return ring + (k * R + r) * (kPlanes * threads) + threadIdx.x; };
  if (VEC && !act)  // threads without columns read zeros
    for (int k = 0; k < kRing * R; ++k)
#pragma unroll
      for (int i = 0; i < kPlanes; ++i) slot(0, k)[i * threads] = make_uint4(0u, 0u, 0u, 0u);
  if (!GL && threadIdx.x < 2 * 2 * R * W) red[threadIdx.x] = 0.f;
  if (!GL) __syncthreads();

  Walk ahead = at;
  auto row_of = [&](const Walk& w, int r) { return w.base + r * kGroups + grp; };
  // bit r: row r of the step is there and no padding
  auto validity = [&](const Walk& w) {
    uint32_t v = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row_of(w, r);
      if (w.more() && row < w.end && (!a.mask || a.mask[row])) v |= 1u << r;
    }
    return v;
  };
  uint32_t valids = 0;  // R bits for each step from the current one on
  uint32_t next_valid = kAhead ? validity(ahead) : 0u;
  int put = 0, get = 0;
  using BX = typename Bits<TX>::type;
  using BB = typename Bits<TB>::type;
  Coming<BX> next_dout, next_o;
  Coming<BB> next_y, next_du;
  auto fetch = [&](int k) {  // the step `ahead` stands at, the k-th to be worked on
    if (ahead.more()) {
      valids |= next_valid << (k * R);
      if (kHeld && (next_valid & 1u)) {
        const long long row = row_of(ahead, 0);
        if (a.dout) next_dout.read(reinterpret_cast<const BX*>(a.dout + row * a.ld_dout), j, n, d);
        if (a.pre) {
          next_o.read(reinterpret_cast<const BX*>(a.o + row * a.ld_o), j, n, d);
          next_du.read(reinterpret_cast<const BB*>(a.du + row * a.ld_du), j, n, d);
        }
        if (with_y) next_y.read(reinterpret_cast<const BB*>(a.y + row * a.ld_y), j, n, d);
      }
#pragma unroll
      for (int r = 0; VEC && r < R; ++r) {
        uint4* to = slot(put, r);
        if (next_valid >> r & 1u) {
          if (act) {
            const long long row = row_of(ahead, r);
            if (a.dout) ring_copy(to, a.dout + row * a.ld_dout + j * kE, threads);
            if (a.pre) {
              ring_copy(to + kPX * threads, a.o + row * a.ld_o + j * kE, threads);
              ring_copy(to + (2 * kPX + kPB) * threads, a.du + row * a.ld_du + j * kE, threads);
            }
            if (with_y) ring_copy(to + 2 * kPX * threads, a.y + row * a.ld_y + j * kE, threads);
          }
        } else if (GL || next_valid) {  // padding beside rows that count
#pragma unroll
          for (int i = 0; i < kPlanes; ++i) to[i * threads] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      ahead.next(kStep);
      next_valid = validity(ahead);
      if (++put == kRing) put = 0;
    }
    if (VEC) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  next_dout.clear(); next_o.clear(); next_y.clear(); next_du.clear();
  if (kAhead)
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k) fetch(k);

  // the statistics of the step that `at` stands at
  float mp[R], rp[R], my[R], ry[R];
  auto statistics = [&](const Walk& w) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row_of(w, r);
      mp[r] = rp[r] = my[r] = ry[r] = 0.f;
      if (w.more() && row < w.end) {
        if (layer_pre) mp[r] = a.m_pre[row];
        if (a.pre) rp[r] = a.r_pre[row];
        if (layer_post) my[r] = a.m_post[row];
        if (a.post) ry[r] = a.r_post[row];
      }
    }
  };
  statistics(at);
  while (at.more()) {
    const int gate_row = at.gate;
    const Walk here = at;
    uint32_t valid;
    Row8<TX> held_dout, held_o;
    Row8<TB> held_y, held_du;
    if (kHeld) {
      held_dout.take(next_dout);
      held_o.take(next_o);
      held_y.take(next_y);
      held_du.take(next_du);
    }
    if (kAhead) {
      fetch(kRing - 1);
      valid = valids & ((1u << R) - 1u);
      valids >>= R;
      if (VEC) asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
    } else {
      valid = validity(at);
    }
    const int ring_at = get;
    if (++get == kRing) get = 0;
    float m0[R], q0[R], m1[R], q1[R];
    if (GL || valid)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool v = valid >> r & 1u;
        q0[r] = v ? rp[r] : 0.f;
        q1[r] = v ? ry[r] : 0.f;
        m0[r] = v ? -mp[r] * q0[r] : 0.f;
        m1[r] = v ? -my[r] * q1[r] : 0.f;
      }
    at.next(kStep);
    statistics(at);
    const bool ends = cut && at.gate != here.gate;  // the last step of a gate row
    const uint32_t present = (row_of(here, R - 1) < here.end ? 1u << (R - 1) : 0u) |
                             (row_of(here, 0) < here.end ? 1u : 0u);
    if (GL || valid) {  // (without groups in warps the whole CTA agrees)
      auto values = [&](auto* base, long long ld, int plane, int r, const auto& held) {
        if (kHeld) return valid & 1u ? held.get() : zero8();
        float v[kE];
        if (VEC) {
          ring_read(slot(ring_at, r) + plane * threads, threads, base, v);
        } else {
#pragma unroll
          for (int i = 0; i < kE; ++i) v[i] = 0.f;
          if (valid >> r & 1u) load<false>(base + row_of(here, r) * ld, j, n, d, v);
        }
        return pairs(v);
      };
      F8 D[R];
#pragma unroll
      for (int r = 0; r < R; ++r) D[r] = a.dout ? values(a.dout, a.ld_dout, 0, r, held_dout) : zero8();
      // columns past d hold 0 in every parameter and input, so that no sum sees what
      // the rest of the arithmetic makes of them
      if (a.pre) {
        F8 oh[R], w[R];
        uint64_t s[R][2];
        float2 c[R];
        const F8 wp = w_pre.get(j, n, d);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          oh[r] = values(a.o, a.ld_o, kPX, r, held_o);
          w[r] = values(a.du, a.ld_du, 2 * kPX + kPB, r, held_du);
          const uint64_t q = pk(q0[r], q0[r]), mq = pk(m0[r], m0[r]);
          s[r][0] = s[r][1] = 0ull;
#pragma unroll
          for (int i = 0; i < kE / 2; ++i) {
            oh[r].p[i] = fma2(oh[r].p[i], q, mq);
            s_wpre.p[i] = fma2(w[r].p[i], oh[r].p[i], s_wpre.p[i]);
            s_bpre.p[i] = add2(s_bpre.p[i], w[r].p[i]);
            w[r].p[i] = mul2(wp.p[i], w[r].p[i]);
            s[r][0] = add2(s[r][0], w[r].p[i]);
            s[r][1] = fma2(w[r].p[i], oh[r].p[i], s[r][1]);
          }
        }
        group_sums<GL, R, W>(s, red, turn, c);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float c0 = layer_pre ? -c[r].x * inv * q0[r] : 0.f, c1 = -c[r].y * inv * q0[r];
          const uint64_t q = pk(q0[r], q0[r]), k0 = pk(c0, c0), k1 = pk(c1, c1);
#pragma unroll
          for (int i = 0; i < kE / 2; ++i)
            D[r].p[i] = add2(D[r].p[i], fma2(w[r].p[i], q, fma2(oh[r].p[i], k1, k0)));
        }
      }
      if (a.dx) {
        const uint64_t sc = pk(a.scale, a.scale);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float t[kE];
          F8 x;
#pragma unroll
          for (int i = 0; i < kE / 2; ++i) x.p[i] = mul2(D[r].p[i], sc);
          singles(x, t);
          if (present >> r & 1u) store<VEC>(a.dx + row_of(here, r) * a.ld_dx, j, n, d, t);
        }
      }
      if (with_y) {
        F8 yn[R], w;
        if (a.post) w = w_post.get(j, n, d);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          yn[r] = values(a.y, a.ld_y, 2 * kPX, r, held_y);
          if (a.post) {
            const uint64_t q = pk(q1[r], q1[r]), mq = pk(m1[r], m1[r]);
#pragma unroll
            for (int i = 0; i < kE / 2; ++i) yn[r].p[i] = fma2(yn[r].p[i], q, mq);
          }
        }
        if (sum_gate) {
          F8 b = zero8();
          if (a.post && a.b_post) b = b_post.get(j, n, d);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            F8 z = yn[r];
            if (a.post)
#pragma unroll
              for (int i = 0; i < kE / 2; ++i) z.p[i] = fma2(w.p[i], yn[r].p[i], b.p[i]);
            if (each) {
              float t[kE];
#pragma unroll
              for (int i = 0; i < kE / 2; ++i) z.p[i] = mul2(D[r].p[i], z.p[i]);
              singles(z, t);
              if (present >> r & 1u) store<VEC>(a.d_gate + (long long)row_of(here, r) * d, j, n, d, t);
            } else {
#pragma unroll
              for (int i = 0; i < kE / 2; ++i) s_gate.p[i] = fma2(D[r].p[i], z.p[i], s_gate.p[i]);
            }
          }
        }
        if (a.gate)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            // 0 for padding, whose gate may hold NaN or infinity: these times 0 are NaN. (A
            // gate row of several tokens is only padding's where no row of a step is valid.)
            const bool v = valid >> r & 1u;
            if (each) gate.set(v ? a.gate + (long long)row_of(here, r) * d : nullptr, j, n, d);
            const F8 t = gate.get(j, n, d, !GL || v);
#pragma unroll
            for (int i = 0; i < kE / 2; ++i) D[r].p[i] = mul2(D[r].p[i], t.p[i]);
          }
        if (a.post) {
          uint64_t s[R][2];
          float2 c[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            s[r][0] = s[r][1] = 0ull;
#pragma unroll
            for (int i = 0; i < kE / 2; ++i) {
              s_wpost.p[i] = fma2(D[r].p[i], yn[r].p[i], s_wpost.p[i]);
              s_bpost.p[i] = add2(s_bpost.p[i], D[r].p[i]);
              D[r].p[i] = mul2(D[r].p[i], w.p[i]);
              s[r][0] = add2(s[r][0], D[r].p[i]);
              s[r][1] = fma2(D[r].p[i], yn[r].p[i], s[r][1]);
            }
          }
          group_sums<GL, R, W>(s, red, turn, c);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float c0 = layer_post ? -c[r].x * inv * q1[r] : 0.f, c1 = -c[r].y * inv * q1[r];
            const uint64_t q = pk(q1[r], q1[r]), k0 = pk(c0, c0), k1 = pk(c1, c1);
#pragma unroll
            for (int i = 0; i < kE / 2; ++i) D[r].p[i] = fma2(D[r].p[i], q, fma2(yn[r].p[i], k1, k0));
          }
        }
        if (a.dy)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            float t[kE];
            singles(D[r], t);
            if (present >> r & 1u) store<VEC>(a.dy + row_of(here, r) * a.ld_dy, j, n, d, t);
          }
      }
    }
    // padding gives 0 (whatever the arithmetic made of zero rows, NaN parameters included)
#pragma unroll
    for (int r = 0; r < R; ++r)
      if ((present & ~valid) >> r & 1u) {
        float t[kE];
#pragma unroll
        for (int i = 0; i < kE; ++i) t[i] = 0.f;
        if (a.dx) store<VEC>(a.dx + row_of(here, r) * a.ld_dx, j, n, d, t);
        if (a.dy) store<VEC>(a.dy + row_of(here, r) * a.ld_dy, j, n, d, t);
        if (sum_gate && each) store<VEC>(a.d_gate + (long long)row_of(here, r) * d, j, n, d, t);
      }
    if (ends) {
      if (sum_gate) flush(s_gate, a.d_gate + (long long)gate_row * d);
      if (a.gate && at.more()) gate.set(a.gate + (long long)at.gate * d, j, n, d);
    }
  }
  float* part = a.part + (long long)blockIdx.x * 4 * d;
  if (a.wanted & 1) flush(s_wpost, part);
  if (a.wanted & 2) flush(s_bpost, part + d);
  if (a.wanted & 4) flush(s_wpre, part + 2 * (long long)d);
  if (a.wanted & 8) flush(s_bpre, part + 3 * (long long)d);
  if (sum_gate && a.pieces > 1) flush(s_gate, a.part_gate + (long long)blockIdx.x * d);
}

// The forward over many rows of bf16, two at a time, the next steps' rows on their way
// to shared memory as in the backward. A CTA takes every gridDim.x-th chunk of rows. 16
// warps on an SM: with 20 or 24 and fewer registers 20,000-odd rows took 2 to 19% longer.
template <typename TX, typename TB>
__host__ __device__ constexpr int stream_steps() {  // of a ring of 320 bytes a thread
  return 320 / (2 * kE * (int)(sizeof(TX) + sizeof(TB)));
}

template <typename TX, typename TB>
__global__ void __launch_bounds__(kThreads, 4)
    forward_stream_kernel(const ForwardArgs<TX, TB> a, const int chunk) {
  constexpr int R = 2, W = kThreads / 32, kRing = stream_steps<TX, TB>();
  constexpr int kPX = kE * sizeof(TX) / 16, kPB = kE * sizeof(TB) / 16, kPlanes = kPX + kPB;
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float red[2 * 2 * R * W];
  const int threads = (int)blockDim.x;
  int turn = 0;
  const int n = threads, j = (int)threadIdx.x;
  const int d = a.d;
  const float inv = 1.f / (float)d;
  const bool act = j * kE < d;
  Param<TB, true> w_post, b_post, w_pre, b_pre, gate[R];
  w_post.set(a.w_post, j, n, d);
  b_post.set(a.b_post, j, n, d);
  w_pre.set(a.w_pre, j, n, d);
  b_pre.set(a.b_pre, j, n, d);
  int gate_at[R] = {0, 0};
  if (a.gate)
#pragma unroll
    for (int r = 0; r < R; ++r) gate[r].set(a.gate, j, n, d);

  auto slot = [&](int k, int r) { return ring + (k * R + r) * (kPlanes * threads) + threadIdx.x; };
  if (!act)  // threads without columns read zeros
    for (int k = 0; k < kRing * R; ++k)
#pragma unroll
      for (int i = 0; i < kPlanes; ++i) slot(0, k)[i * threads] = make_uint4(0u, 0u, 0u, 0u);
  if (threadIdx.x < 2 * 2 * R * W) red[threadIdx.x] = 0.f;
  __syncthreads();

  Walk at;
  at.cut = false;
  at.gate = 0;
  at.last = a.T;
  at.size = chunk;
  at.base = (int)min((long long)a.T, (long long)blockIdx.x * chunk);
  at.skip = (int)min((long long)a.T, (long long)(gridDim.x - 1) * chunk);
  at.end = min(at.last - at.base, chunk) + at.base;
  Walk ahead = at;
  auto row_of = [&](const Walk& w, int r) { return w.base + r; };
  auto validity = [&](const Walk& w) {
    uint32_t v = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row_of(w, r);
      if (w.more() && row < w.end && (!a.mask || a.mask[row])) v |= 1u << r;
    }
    return v;
  };
  uint32_t valids = 0, next_valid = validity(ahead);
  int put = 0, get = 0;
  auto fetch = [&](int k) {
    if (ahead.more()) {
      valids |= next_valid << (k * R);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint4* to = slot(put, r);
        if (next_valid >> r & 1u) {
          if (act) {
            const long long row = row_of(ahead, r);
            ring_copy(to, a.x + row * a.ld_x + j * kE, threads);
            if (a.y) ring_copy(to + kPX * threads, a.y + row * a.ld_y + j * kE, threads);
          }
        } else if (next_valid) {
#pragma unroll
          for (int i = 0; i < kPlanes; ++i) to[i * threads] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      ahead.next(R);
      next_valid = validity(ahead);
      if (++put == kRing) put = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int k = 0; k < kRing - 1; ++k) fetch(k);

  // v to w (v - mean) rstd + b, for the step's rows together
  auto norm_rows = [&](F8 (&v)[R], int kind, const Param<TB, true>& w, const Param<TB, true>& b,
                       const TB* bias, float (&mean)[R], float (&rstd)[R]) {
    uint64_t s[R][2];
    float2 c[R];
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = 0.f;
    if (kind == UNIF_MOE_NORM_LAYER) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        s[r][0] = add2(add2(v[r].p[0], v[r].p[1]), add2(v[r].p[2], v[r].p[3]));
        s[r][1] = 0ull;
      }
      group_sums<0, R, W>(s, red, turn, c);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        mean[r] = c[r].x * inv;
        const float m = act ? -mean[r] : 0.f;
#pragma unroll
        for (int i = 0; i < kE / 2; ++i) v[r].p[i] = add2(v[r].p[i], pk(m, m));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r][0] = s[r][1] = 0ull;
#pragma unroll
      for (int i = 0; i < kE / 2; ++i) s[r][0] = fma2(v[r].p[i], v[r].p[i], s[r][0]);
    }
    group_sums<0, R, W>(s, red, turn, c);
    const F8 wv = w.get(j, n, d);
    F8 bv = zero8();
    if (bias) bv = b.get(j, n, d);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rstd[r] = rsqrtf(c[r].x * inv + a.eps);
#pragma unroll
      for (int i = 0; i < kE / 2; ++i)
        v[r].p[i] = fma2(mul2(v[r].p[i], pk(rstd[r], rstd[r])), wv.p[i], bv.p[i]);
    }
  };
  while (at.more()) {
    const Walk here = at;
    if (a.gate && a.gate_rows)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int g = min(row_of(here, r), a.T - 1) / a.gate_rows;
        if (g != gate_at[r]) {
          gate[r].set(a.gate + (long long)g * d, j, n, d);
          gate_at[r] = g;
        }
      }
    fetch(kRing - 1);
    const uint32_t valid = valids & ((1u << R) - 1u);
    valids >>= R;
    asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
    const int ring_at = get;
    if (++get == kRing) get = 0;
    at.next(R);
    const uint32_t present = (row_of(here, 1) < here.end ? 2u : 0u) | (row_of(here, 0) < here.end ? 1u : 0u);
    float m1[R], r1[R], m2[R], r2[R];
    if (valid) {  // (the whole CTA agrees)
      F8 o[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float t[kE];
        ring_read(slot(ring_at, r), threads, a.x, t);
        o[r] = pairs(t);
      }
      if (a.y) {
        F8 z[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float t[kE];
          ring_read(slot(ring_at, r) + kPX * threads, threads, a.y, t);
          z[r] = pairs(t);
        }
        if (a.post) norm_rows(z, a.post, w_post, b_post, a.b_post, m1, r1);
        const uint64_t sc = pk(a.scale, a.scale);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (a.gate) {
            const F8 g = gate[r].get(j, n, d);
#pragma unroll
            for (int i = 0; i < kE / 2; ++i) z[r].p[i] = mul2(z[r].p[i], g.p[i]);
          }
#pragma unroll
          for (int i = 0; i < kE / 2; ++i) o[r].p[i] = fma2(o[r].p[i], sc, z[r].p[i]);
          if (a.out && (valid >> r & 1u)) {
            float t[kE];
            singles(o[r], t);
            store<true>(a.out + row_of(here, r) * a.ld_out, j, n, d, t);
          }
        }
      }
      if (a.pre) {
        norm_rows(o, a.pre, w_pre, b_pre, a.b_pre, m2, r2);
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (valid >> r & 1u) {
            float t[kE];
            singles(o[r], t);
            store<true>(a.u + row_of(here, r) * a.ld_u, j, n, d, t);
          }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!(present >> r & 1u)) continue;
      const bool v = valid >> r & 1u;
      const int row = row_of(here, r);
      if (!v) {  // padding gives 0
        float t[kE];
#pragma unroll
        for (int i = 0; i < kE; ++i) t[i] = 0.f;
        if (a.y && a.out) store<true>(a.out + row * a.ld_out, j, n, d, t);
        if (a.pre) store<true>(a.u + row * a.ld_u, j, n, d, t);
      }
      if (j == 0) {
        if (a.y && a.post) {
          if (a.m_post) a.m_post[row] = v ? m1[r] : 0.f;
          if (a.r_post) a.r_post[row] = v ? r1[r] : 0.f;
        }
        if (a.pre) {
          if (a.m_pre) a.m_pre[row] = v ? m2[r] : 0.f;
          if (a.r_pre) a.r_pre[row] = v ? r2[r] : 0.f;
        }
      }
    }
  }
}

struct FinishArgs {
  int d, ctas, pieces, gates;  // gates: gate rows whose pieces are added here
  int sums;                    // 4, and the gate row where there is one: sums over all CTAs
  const float* part;
  const float* part_gate;
  float* to[4];   // dw_post, db_post, dw_pre, db_pre
  float* d_gate;
};

// The first CTAs: 32 columns of one of the sums over all CTAs each, 32 threads per
// column add every 32nd CTA's share and a tree adds those. The others, with several
// gate rows: a thread per column of a gate row adds its pieces.
__global__ void __launch_bounds__(1024) finish_kernel(const FinishArgs a) {
  __shared__ float t[32][33];
  grid_dep_wait();
  const int tiles = (a.d + 31) / 32;
  if ((int)blockIdx.x < a.sums * tiles) {
    const int k = blockIdx.x / tiles, c0 = (blockIdx.x - k * tiles) * 32;
    float* to = k == 0 ? a.to[0] : k == 1 ? a.to[1] : k == 2 ? a.to[2] : k == 3 ? a.to[3] : a.d_gate;
    if (!to) return;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = c0 + x;
    const float* from = k < 4 ? a.part + (long long)k * a.d + c : a.part_gate + c;
    const long long step = k < 4 ? 4ll * a.d : a.d;
    float s = 0.f;
    if (c < a.d)
#pragma unroll 8
      for (int i = y; i < a.ctas; i += 32) s += from[i * step];
    t[y][x] = s;
    __syncthreads();
    s = t[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (x == 0 && c0 + y < a.d) to[c0 + y] = s;
    return;
  }
  const long long i = (long long)(blockIdx.x - a.sums * tiles) * 1024 + threadIdx.x;
  const int g = (int)(i / a.d), c = (int)(i - (long long)g * a.d);
  if (g >= a.gates) return;
  const float* from = a.part_gate + (long long)g * a.pieces * a.d + c;
  float s = 0.f;
#pragma unroll 4
  for (int k = 0; k < a.pieces; ++k) s += from[(long long)k * a.d];
  a.d_gate[i] = s;
}

// ---- host ----
// Lanes of a row's group within a warp, or 0 where a row takes a CTA.
inline int group_lanes(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : d <= 256 ? 32 : 0; }
inline int cta_threads(int d) {
  return group_lanes(d) ? kThreads : (d + 32 * kE - 1) / (32 * kE) * 32;
}

struct Plan {
  int run, pieces, ctas;
};

// How the backward's rows are split. Where a gate row's rows are many, they are
// dealt out in chunks to the same number of CTAs for every gate row; where they
// are few, a CTA's run holds whole gate rows. About as many CTAs as fit on the
// SMs, each with enough rows that its column sums are worth writing.
Plan plan_backward(const unif_moe_block_norm* p, bool gate, int sms) {
  const int warps = cta_threads(p->width) / 32;
  const int groups = group_lanes(p->width) ? kThreads / group_lanes(p->width) : 1;
  const int slots = sms * (warps > 12 ? 1 : 12 / warps);
  const long long T = p->tokens;
  const long long period = gate && p->gate_rows && p->gate_rows < T ? p->gate_rows : T;
  const long long G = (T + period - 1) / period;
  const long long chunk = groups < 2 ? 4 : 2ll * groups;  // whole steps of 1 or 2 rows a group
  long long want = (T + slots - 1) / slots;
  if (want < 8ll * groups) want = 8ll * groups;
  Plan r;
  if (period > want) {
    long long pieces = slots / G < 1 ? 1 : slots / G;
    const long long most = period / want;
    if (pieces > most) pieces = most;
    r.pieces = (int)pieces;
    r.run = pieces > 1 ? (int)chunk : (int)period;
    r.ctas = (int)(G * r.pieces);
  } else {
    r.pieces = 1;
    r.run = (int)(want / period * period);
    r.ctas = (int)((T + r.run - 1) / r.run);
  }
  return r;
}

template <typename T>
bool vec_ok(const T* p, long long ld) {
  return reinterpret_cast<uintptr_t>(p) % (kE * sizeof(T)) == 0 && ld % kE == 0;
}

template <typename TX, typename TB>
cudaError_t launch_stream(const ForwardArgs<TX, TB>& a, int threads, int sms, cudaStream_t s) {
  const int smem = stream_steps<TX, TB>() * 2 * kE * (int)(sizeof(TX) + sizeof(TB)) * threads;
  constexpr int chunk = 4;  // two steps
  const long long chunks = ((long long)a.T + chunk - 1) / chunk;
  const int most = sms * (512 / threads);
  forward_stream_kernel<TX, TB><<<(unsigned)(chunks < most ? chunks : most), threads, smem, s>>>(a, chunk);
  return cudaGetLastError();
}

template <typename TX, typename TB, bool VEC>
cudaError_t launch_fwd(const ForwardArgs<TX, TB>& a, int sms, cudaStream_t s) {
  const int threads = cta_threads(a.d);
  // A bf16 stream of 257 to 1,024 columns: forward_stream_kernel once every SM has 16
  // rows. us, a row to a group of threads against it, both norms: 64 rows an SM, 9,728 x 384
  // 12.4 and 10.1, x 1,024 22.1 and 18.5; 16 rows an SM, 2,432 x 384 4.8 and 4.7, x 640 5.8 and
  // 5.2, x 1,024 7.4 and 6.6; 8 rows an SM, 1,216 x 384 4.0 and 4.1, x 640 4.3 and 4.5, x 1,024
  // 4.5 and 4.6. Other widths: 9,728 x 2,048 39.7 and 41.6; 77,824 x 80 16.9 and 16.1, 19,456 x
  // 80 5.1 and 5.5. An fp32 stream has more bytes for the same work and more CTAs hide them better: 9,728 x 1,024
  // over bf16 23.6 and 27.4.
  if constexpr (VEC && sizeof(TX) == 2)
    if (!group_lanes(a.d) && threads <= kThreads && a.T >= 16ll * sms)
      return launch_stream(a, threads, sms, s);
  switch (group_lanes(a.d)) {
    case 8: forward_kernel<TX, TB, VEC, 8, kThreads><<<(a.T + 15) / 16, threads, 0, s>>>(a); break;
    case 16: forward_kernel<TX, TB, VEC, 16, kThreads><<<(a.T + 7) / 8, threads, 0, s>>>(a); break;
    case 32: forward_kernel<TX, TB, VEC, 32, kThreads><<<(a.T + 3) / 4, threads, 0, s>>>(a); break;
    default:
      if (VEC) forward_kernel<TX, TB, true, 0, 1024><<<a.T, threads, 0, s>>>(a);
      else if (threads <= 64) forward_kernel<TX, TB, false, 0, 64><<<a.T, 64, 0, s>>>(a);
      else if (threads <= 128) forward_kernel<TX, TB, false, 0, 128><<<a.T, 128, 0, s>>>(a);
      else if (threads <= 256) forward_kernel<TX, TB, false, 0, 256><<<a.T, 256, 0, s>>>(a);
      else if (threads <= 384) forward_kernel<TX, TB, false, 0, 384><<<a.T, 384, 0, s>>>(a);
      else if (threads <= 512) forward_kernel<TX, TB, false, 0, 512><<<a.T, 512, 0, s>>>(a);
      else forward_kernel<TX, TB, false, 0, 1024><<<a.T, 1024, 0, s>>>(a);
      break;
  }
  return cudaGetLastError();
}

template <typename TX, typename TB, bool VEC, int GL, int MT>
cudaError_t launch_bwd_as(const BackwardArgs<TX, TB>& a, int ctas, int threads, cudaStream_t s) {
  const int smem = VEC ? ring_steps<TX, TB>(MT) * step_rows(true, MT) * row_bytes<TX, TB>() * threads : 0;
  if (smem > 40 * 1024) {  // with the static part above what needs no leave
    const cudaError_t e = allow_smem_once(backward_kernel<TX, TB, VEC, GL, MT>, smem);
    if (e != cudaSuccess) return e;
  }
  backward_kernel<TX, TB, VEC, GL, MT><<<ctas, threads, smem, s>>>(a);
  return cudaGetLastError();
}

template <typename TX, typename TB, bool VEC>
cudaError_t launch_bwd(const BackwardArgs<TX, TB>& a, int ctas, cudaStream_t s) {
  const int threads = cta_threads(a.d);
  switch (group_lanes(a.d)) {
    case 8: return launch_bwd_as<TX, TB, VEC, 8, kThreads>(a, ctas, threads, s);
    case 16: return launch_bwd_as<TX, TB, VEC, 16, kThreads>(a, ctas, threads, s);
    case 32: return launch_bwd_as<TX, TB, VEC, 32, kThreads>(a, ctas, threads, s);
  }
  // (without VEC the kernel counts on all of its threads)
  if constexpr (!VEC) {
    if (threads <= 64) return launch_bwd_as<TX, TB, false, 0, 64>(a, ctas, 64, s);
    if (threads > 128 && threads <= 256) return launch_bwd_as<TX, TB, false, 0, 256>(a, ctas, 256, s);
  }
  if (threads <= 128) return launch_bwd_as<TX, TB, VEC, 0, 128>(a, ctas, VEC ? threads : 128, s);
  if (threads <= 384) return launch_bwd_as<TX, TB, VEC, 0, 384>(a, ctas, VEC ? threads : 384, s);
  if (threads <= 512) return launch_bwd_as<TX, TB, VEC, 0, 512>(a, ctas, VEC ? threads : 512, s);
  // still wider rows: no room for a ring beside 1,024 threads
  return launch_bwd_as<TX, TB, false, 0, 1024>(a, ctas, 1024, s);
}

int check_desc(const unif_moe_block_norm* p) {
  if (!p) { set_error("the description is NULL"); return UNIF_MOE_ERR_ARG; }
  if (p->tokens < 0 || p->width < 1 || p->gate_rows < 0) {
    set_error("bad sizes: tokens=%d width=%d gate_rows=%d", p->tokens, p->width, p->gate_rows);
    return UNIF_MOE_ERR_ARG;
  }
  if (p->tokens > UNIF_MOE_NORM_MAX_TOKENS) {
    set_error("tokens=%d above %d", p->tokens, UNIF_MOE_NORM_MAX_TOKENS);
    return UNIF_MOE_ERR_SHAPE;
  }
  if (p->width > UNIF_MOE_NORM_MAX_WIDTH) {
    set_error("width=%d above %d", p->width, UNIF_MOE_NORM_MAX_WIDTH);
    return UNIF_MOE_ERR_SHAPE;
  }
  auto type = [](int t) { return t == UNIF_MOE_F32 || t == UNIF_MOE_BF16; };
  if (!type(p->stream_dtype) || !type(p->branch_dtype) ||
      (p->stream_dtype == UNIF_MOE_BF16 && p->branch_dtype == UNIF_MOE_F32)) {
    set_error("bad dtypes: stream %d, branch %d (a bf16 stream takes a bf16 branch)",
              p->stream_dtype, p->branch_dtype);
    return UNIF_MOE_ERR_ARG;
  }
  auto kind = [](int k) { return k >= UNIF_MOE_NORM_NONE && k <= UNIF_MOE_NORM_RMS; };
  if (!kind(p->post_norm) || !kind(p->pre_norm)) {
    set_error("bad norms: post %d, pre %d", p->post_norm, p->pre_norm);
    return UNIF_MOE_ERR_ARG;
  }
  if (!(p->eps >= 0.f) || !isfinite(p->eps) || !isfinite(p->res_scale)) {
    set_error("eps must be finite and >= 0, res_scale finite");
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

bool ld_bad(const void* p, long long ld, int d) { return p && ld < d; }

template <typename TX, typename TB>
cudaError_t forward_as(const unif_moe_block_norm* p, int sms, const void* x, long long ld_x, const void* y,
                       long long ld_y, const uint8_t* mask, const void* w_post, const void* b_post,
                       const void* gate, const void* w_pre, const void* b_pre, void* out,
                       long long ld_out, void* u, long long ld_u, float* m_post, float* r_post,
                       float* m_pre, float* r_pre, cudaStream_t s) {
  ForwardArgs<TX, TB> a{p->tokens, p->width, p->post_norm, p->pre_norm, p->gate_rows,
                        p->res_scale, p->eps,
                        static_cast<const TX*>(x), static_cast<const TB*>(y),
                        ld_x, ld_y, ld_out, ld_u, mask,
                        static_cast<const TB*>(w_post), static_cast<const TB*>(b_post),
                        static_cast<const TB*>(gate), static_cast<const TB*>(w_pre),
                        static_cast<const TB*>(b_pre), static_cast<TX*>(out),
                        static_cast<TB*>(u), m_post, r_post, m_pre, r_pre};
  const bool vec = p->width % kE == 0 && vec_ok(a.x, ld_x) && (!y || vec_ok(a.y, ld_y)) &&
                   (!out || vec_ok(a.out, ld_out)) && (!u || vec_ok(a.u, ld_u)) &&
                   vec_ok(a.w_post, 0) && vec_ok(a.b_post, 0) && vec_ok(a.gate, 0) &&
                   vec_ok(a.w_pre, 0) && vec_ok(a.b_pre, 0);
  return vec ? launch_fwd<TX, TB, true>(a, sms, s) : launch_fwd<TX, TB, false>(a, sms, s);
}

int64_t workspace_floats(const Plan& pl, int d) {
  return (int64_t)pl.ctas * d * (pl.pieces > 1 ? 5 : 4);
}

template <typename TX, typename TB>
cudaError_t backward_as(const unif_moe_block_norm* p, const Plan& pl, const void* o, long long ld_o,
                        const void* y, long long ld_y, const uint8_t* mask, const void* w_post,
                        const void* b_post, const void* gate, const void* w_pre,
                        const float* m_post, const float* r_post, const float* m_pre,
                        const float* r_pre, const void* dout, long long ld_dout, const void* du,
                        long long ld_du, void* dx, long long ld_dx, void* dy, long long ld_dy,
                        float* const (&to)[4], float* d_gate, float* ws, cudaStream_t s) {
  BackwardArgs<TX, TB> a{};
  a.T = p->tokens; a.d = p->width; a.post = p->post_norm; a.pre = p->pre_norm;
  a.gate_rows = gate ? p->gate_rows : 0;
  a.scale = y ? p->res_scale : 1.f;
  a.o = static_cast<const TX*>(o); a.y = static_cast<const TB*>(y);
  a.dout = static_cast<const TX*>(dout); a.du = static_cast<const TB*>(du);
  a.ld_o = ld_o; a.ld_y = ld_y; a.ld_dout = ld_dout; a.ld_du = ld_du; a.ld_dx = ld_dx; a.ld_dy = ld_dy;
  a.mask = mask;
  a.w_post = static_cast<const TB*>(w_post); a.b_post = static_cast<const TB*>(b_post);
  a.gate = static_cast<const TB*>(gate); a.w_pre = static_cast<const TB*>(w_pre);
  a.m_post = m_post; a.r_post = r_post; a.m_pre = m_pre; a.r_pre = r_pre;
  a.dx = static_cast<TX*>(dx); a.dy = static_cast<TB*>(dy); a.d_gate = d_gate;
  a.part = ws;
  a.part_gate = ws + (int64_t)pl.ctas * 4 * a.d;
  for (int i = 0; i < 4; ++i) a.wanted |= to[i] ? 1 << i : 0;
  a.wanted |= d_gate ? 16 : 0;
  a.pieces = pl.pieces; a.run = pl.run;
  auto ok = [](const auto* q, long long ld) { return !q || vec_ok(q, ld); };
  // d_gate is written a gate row at a time by the CTA that holds it
  const bool vec = a.d % kE == 0 && ok(a.o, ld_o) && ok(a.y, ld_y) && ok(a.dout, ld_dout) &&
                   ok(a.du, ld_du) && ok(a.dx, ld_dx) && ok(a.dy, ld_dy) && ok(a.w_post, 0) &&
                   ok(a.b_post, 0) && ok(a.gate, 0) && ok(a.w_pre, 0) && ok(d_gate, 0) && ok(ws, 0);
  cudaError_t e = vec ? launch_bwd<TX, TB, true>(a, pl.ctas, s)
                      : launch_bwd<TX, TB, false>(a, pl.ctas, s);
  const bool gates = d_gate && pl.pieces > 1;
  if (e != cudaSuccess || !((a.wanted & 15) || gates)) return e;
  const int gate_rows = gates ? pl.ctas / pl.pieces : 0;
  const int sums = gate_rows == 1 ? 5 : 4;
  FinishArgs f{a.d, pl.ctas, pl.pieces, gate_rows, sums, a.part, a.part_gate,
               {to[0], to[1], to[2], to[3]}, d_gate};
  const long long more = gate_rows > 1 ? ((long long)gate_rows * a.d + 1023) / 1024 : 0;
  return launch_dependent(finish_kernel, dim3((unsigned)(sums * ((a.d + 31) / 32) + more)), dim3(1024),
                          0, s, f);
}

}  // namespace norm
}  // namespace unif

using unif::set_error;
namespace nm = unif::norm;

extern "C" {

int unif_moe_block_norm_forward(const unif_moe_block_norm* p, const void* x, int64_t ld_x,
                                const void* y, int64_t ld_y, const uint8_t* mask,
                                const void* w_post, const void* b_post, const void* gate,
                                const void* w_pre, const void* b_pre, void* out, int64_t ld_out,
                                void* u, int64_t ld_u, float* m_post, float* r_post, float* m_pre,
                                float* r_pre, void* stream) {
  set_error("%s", "");
  const int rc = nm::check_desc(p);
  if (rc != UNIF_MOE_OK) return rc;
  if (p->tokens == 0) return UNIF_MOE_OK;
  if (!y && (p->post_norm || gate || out)) {
    set_error("without y there is no post norm, no gate and no out");
    return UNIF_MOE_ERR_ARG;
  }
  if ((p->post_norm && !w_post) || (p->pre_norm && !w_pre)) {
    set_error("a norm's weight is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (!x || (y && !out && !p->pre_norm) || (p->pre_norm && !u) || (!y && !p->pre_norm)) {
    set_error("x, out or u is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (nm::ld_bad(x, ld_x, p->width) || nm::ld_bad(y, ld_y, p->width) ||
      nm::ld_bad(out, ld_out, p->width) || nm::ld_bad(p->pre_norm ? u : nullptr, ld_u, p->width)) {
    set_error("a row stride is below the width");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
#define UNIF_ARGS p, sms, x, ld_x, y, ld_y, mask, w_post, b_post, gate, w_pre, b_pre, out, ld_out, u, \
                  ld_u, m_post, r_post, m_pre, r_pre, s
  if (p->branch_dtype == UNIF_MOE_F32) e = nm::forward_as<float, float>(UNIF_ARGS);
  else if (p->stream_dtype == UNIF_MOE_F32) e = nm::forward_as<float, __nv_bfloat16>(UNIF_ARGS);
  else e = nm::forward_as<__nv_bfloat16, __nv_bfloat16>(UNIF_ARGS);
#undef UNIF_ARGS
  if (e != cudaSuccess) {
    set_error("block norm forward: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

int64_t unif_moe_block_norm_workspace(const unif_moe_block_norm* p, int gate) {
  set_error("%s", "");
  int sms = 0;
  if (nm::check_desc(p) != UNIF_MOE_OK || unif::sm_count(&sms) != UNIF_MOE_OK) return -1;
  if (p->tokens == 0) return 0;
  return nm::workspace_floats(nm::plan_backward(p, gate != 0, sms), p->width) * (int64_t)sizeof(float);
}

int unif_moe_block_norm_backward(const unif_moe_block_norm* p, const void* out, int64_t ld_out,
                                 const void* y, int64_t ld_y, const uint8_t* mask,
                                 const void* w_post, const void* b_post, const void* gate,
                                 const void* w_pre, const float* m_post, const float* r_post,
                                 const float* m_pre, const float* r_pre, const void* dout,
                                 int64_t ld_dout, const void* du, int64_t ld_du, void* dx,
                                 int64_t ld_dx, void* dy, int64_t ld_dy, float* dw_post,
                                 float* db_post, float* d_gate, float* dw_pre, float* db_pre,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
  set_error("%s", "");
  const int rc = nm::check_desc(p);
  if (rc != UNIF_MOE_OK) return rc;
  const int d = p->width;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  float* const to[4] = {dw_post, db_post, dw_pre, db_pre};
  if (p->tokens == 0) {
    for (float* t : to)
      if (t && cudaMemsetAsync(t, 0, sizeof(float) * d, s) != cudaSuccess) {
        set_error("block norm backward: clearing the gradients failed");
        return UNIF_MOE_ERR_CUDA;
      }
    // one gate row where all tokens share it; none where each has its own
    if (d_gate && p->gate_rows == 0 && cudaMemsetAsync(d_gate, 0, sizeof(float) * d, s) != cudaSuccess) {
      set_error("block norm backward: clearing the gradients failed");
      return UNIF_MOE_ERR_CUDA;
    }
    return UNIF_MOE_OK;
  }
  if (!y && (p->post_norm || gate || dy || d_gate)) {
    set_error("without y there is no post norm, no gate and no dy");
    return UNIF_MOE_ERR_ARG;
  }
  if ((p->post_norm && !w_post) || (p->pre_norm && !w_pre) || (d_gate && !gate) ||
      ((dw_post || db_post) && !p->post_norm) || ((dw_pre || db_pre) && !p->pre_norm)) {
    set_error("a norm's weight or the gate is NULL, or a gradient of a norm that is not there is asked for");
    return UNIF_MOE_ERR_ARG;
  }
  const bool layer_post = p->post_norm == UNIF_MOE_NORM_LAYER;
  const bool layer_pre = p->pre_norm == UNIF_MOE_NORM_LAYER;
  if ((p->pre_norm && (!out || !du || !r_pre)) || (layer_pre && !m_pre) ||
      (p->post_norm && !r_post) || (layer_post && !m_post) || !(dout || du)) {
    set_error("out, du, dout or a statistic that the norms need is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (nm::ld_bad(p->pre_norm ? out : nullptr, ld_out, d) || nm::ld_bad(y, ld_y, d) ||
      nm::ld_bad(dout, ld_dout, d) || nm::ld_bad(p->pre_norm ? du : nullptr, ld_du, d) ||
      nm::ld_bad(dx, ld_dx, d) || nm::ld_bad(dy, ld_dy, d)) {
    set_error("a row stride is below the width");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  const nm::Plan pl = nm::plan_backward(p, gate != nullptr, sms);
  const int64_t need = nm::workspace_floats(pl, d) * (int64_t)sizeof(float);
  if (need > workspace_bytes || !workspace) {
    set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (reinterpret_cast<uintptr_t>(workspace) & 15u) {
    set_error("the workspace must be 16-byte aligned");
    return UNIF_MOE_ERR_ARG;
  }
  cudaError_t e;
#define UNIF_ARGS p, pl, p->pre_norm ? out : nullptr, ld_out, y, ld_y, mask, w_post, b_post, gate, \
                  w_pre, m_post, r_post, m_pre, r_pre, dout, ld_dout, p->pre_norm ? du : nullptr, \
                  ld_du, dx, ld_dx, dy, ld_dy, to, d_gate, static_cast<float*>(workspace), s
  if (p->branch_dtype == UNIF_MOE_F32) e = nm::backward_as<float, float>(UNIF_ARGS);
  else if (p->stream_dtype == UNIF_MOE_F32) e = nm::backward_as<float, __nv_bfloat16>(UNIF_ARGS);
  else e = nm::backward_as<__nv_bfloat16, __nv_bfloat16>(UNIF_ARGS);
#undef UNIF_ARGS
  if (e != cudaSuccess) {
    set_error("block norm backward: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

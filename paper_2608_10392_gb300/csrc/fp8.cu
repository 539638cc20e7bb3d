// Rows to 8-bit floating point under a scale of their own, and back (unif_moe_fp8_quantize /
// _dequantize; fp8.cuh has the rule).
//
// Bound by memory: a row is read once and held in registers while its largest value is
// found, by a warp up to 1,024 columns, by a CTA up to 8,192; wider rows are read twice. (us, at the floor
// of the bytes in brackets: 65,536 x 1,024 fp32 47.2 (49.4: some of them stay in L2), bf16 29.7 (29.7), 12,608 x
// 4,096 fp32 39.7 (38.0), bf16 31.8 (22.8); back to bf16 65,536 x 1,024 36.0 (29.7).)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "fp8.cuh"
#include "internal.cuh"
#include "overlap.h"

namespace unif {
namespace fp8 {

constexpr int kThreads = 256, kPieces = 4;  // pieces of eight values of a thread

template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
  if (VEC) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
    if (left > 0) {
      a = *reinterpret_cast<const float4*>(p);
      b = *(reinterpret_cast<const float4*>(p) + 1);
    }
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int left, float (&v)[8]) {
  if (VEC) {
    uint4 a = make_uint4(0u, 0u, 0u, 0u);
    if (left > 0) a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? __bfloat162float(p[i]) : 0.f;
  }
}

// WARP: a row to a warp, else to the CTA. Thread j of a row's n takes the pieces j, j + n, ...
template <typename T, bool VEC, bool WARP>
__global__ void __launch_bounds__(kThreads)
    quantize_kernel(const T* x, long long rows, int cols, long long ld, uint8_t* codes, long long ld_c,
                    float* scales) {
  __shared__ uint32_t red[kThreads / 32];
  grid_dep_wait();
  const int n = WARP ? 32 : kThreads, j = WARP ? threadIdx.x & 31 : threadIdx.x;
  const long long row = WARP ? (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP && row >= rows) return;
  const T* p = x + row * ld;
  const int pieces = (cols + 7) / 8;
  float v[kPieces][8];
  uint32_t most = 0;
  auto at = [&](int k, int from) { return (from + k * n + j) * 8; };
  auto read = [&](int from) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) load8<VEC>(p + at(k, from), cols - at(k, from), v[k]);
  };
  for (int from = 0; from < pieces; from += kPieces * n) {
    read(from);
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[k][i]));
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (!WARP) {
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) most = max(most, red[w]);
  }
  float by;
  const float scale = row_scale(most, by);
  if (j == 0) scales[row] = scale;
  uint8_t* to = codes + row * ld_c;
  for (int from = 0; from < pieces; from += kPieces * n) {
    if (pieces > kPieces * n) read(from);  // (a row that the registers did not hold)
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int c = at(k, from);
      if (c >= cols) continue;
      const uint2 q = codes8(v[k], by);
      if (VEC) {
        *reinterpret_cast<uint2*>(to + c) = q;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) to[c + i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
      }
    }
  }
}

__device__ __forceinline__ void values2(uint32_t code, float& lo, float& hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  lo = f.x;
  hi = f.y;
}

// Pieces of eight values, numbered row by row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
    dequantize_kernel(const uint8_t* codes, long long ld_c, const float* scales, long long total, int per_row,
                      int cols, T* x, long long ld) {
  grid_dep_wait();
  const long long step = (long long)gridDim.x * kThreads;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
    const long long row = i / per_row;
    const int c = (int)(i - row * per_row) * 8;
    const uint8_t* p = codes + row * ld_c + c;
    const float s = scales[row];
    uint2 q = make_uint2(0u, 0u);
    if (VEC) {
      q = *reinterpret_cast<const uint2*>(p);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < cols) (k < 4 ? q.x : q.y) |= (uint32_t)p[k] << (8 * (k & 3));
    }
    float v[8];
    values2(q.x & 0xffffu, v[0], v[1]);
    values2(q.x >> 16, v[2], v[3]);
    values2(q.y & 0xffffu, v[4], v[5]);
    values2(q.y >> 16, v[6], v[7]);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= s;
    T* o = x + row * ld + c;
    if constexpr (sizeof(T) == 2) {
      if (VEC) {
        uint32_t h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
          h[k] = *reinterpret_cast<const uint32_t*>(&t);
        }
        *reinterpret_cast<uint4*>(o) = make_uint4(h[0], h[1], h[2], h[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < cols) o[k] = __float2bfloat16_rn(v[k]);
      }
    } else if (VEC) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < cols) o[k] = v[k];
    }
  }
}

template <typename T>
cudaError_t quantize(const void* x, long long rows, int cols, long long ld, uint8_t* codes, long long ld_c,
                     float* scales, bool vec, cudaStream_t s) {
  const T* p = static_cast<const T*>(x);
  const bool warp = cols <= 8 * kPieces * 32;
  void (*kernel)(const T*, long long, int, long long, uint8_t*, long long, float*) =
      warp ? (vec ? quantize_kernel<T, true, true> : quantize_kernel<T, false, true>)
           : (vec ? quantize_kernel<T, true, false> : quantize_kernel<T, false, false>);
  const long long grid = warp ? (rows + kThreads / 32 - 1) / (kThreads / 32) : rows;
  return launch_dependent(kernel, dim3((unsigned)grid), dim3(kThreads), 0, s, p, rows, cols, ld, codes, ld_c,
                          scales);
}

template <typename T>
cudaError_t dequantize(const uint8_t* codes, long long ld_c, const float* scales, long long rows, int cols,
                       void* x, long long ld, bool vec, int sms, cudaStream_t s) {
  const int per_row = (cols + 7) / 8;
  const long long total = rows * per_row;
  const long long grid = std::min<long long>((total + kThreads - 1) / kThreads, 32ll * sms);
  void (*kernel)(const uint8_t*, long long, const float*, long long, int, int, T*, long long) =
      vec ? dequantize_kernel<T, true> : dequantize_kernel<T, false>;
  return launch_dependent(kernel, dim3((unsigned)grid), dim3(kThreads), 0, s, codes, ld_c, scales, total,
                          per_row, cols, static_cast<T*>(x), ld);
}

int check(const void* x, int dtype, int64_t rows, int cols, int64_t ld, const void* codes, int64_t ld_c,
          const void* scales) {
  if (rows < 0 || rows > 0x7fffffff - 1024 || cols < 1 || cols > UNIF_MOE_LINEAR_MAX_COLS) {
    set_error("bad sizes: rows=%lld cols=%d", (long long)rows, cols);
    return UNIF_MOE_ERR_ARG;
  }
  if (dtype != UNIF_MOE_F32 && dtype != UNIF_MOE_BF16) {
    set_error("bad dtype %d", dtype);
    return UNIF_MOE_ERR_ARG;
  }
  if (rows > 0 && (!x || !codes || !scales)) {
    set_error("x, codes or scales is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (ld < cols || ld_c < cols) {
    set_error("a row stride is below cols=%d", cols);
    return UNIF_MOE_ERR_ARG;
  }
  // (rows of other CTAs, or later pieces of a row, are still to be read when the first result is written)
  const int64_t size = dtype == UNIF_MOE_F32 ? 4 : 2;
  const Block bx{x, ld * size, cols * size, rows}, bc{codes, ld_c, cols, rows}, bs = flat(scales, rows * 4);
  if (overlap_any(bx, {bc, bs}) || overlap(bc, bs)) {
    set_error("x, codes and scales overlap");
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

// Whether pieces of eight can be moved whole.
bool whole(const void* x, int dtype, int cols, int64_t ld, const void* codes, int64_t ld_c) {
  return cols % 8 == 0 && ld % 8 == 0 && ld_c % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0 &&
         reinterpret_cast<uintptr_t>(codes) % 8 == 0;
}

}  // namespace fp8
}  // namespace unif

using unif::set_error;
namespace f8 = unif::fp8;

extern "C" {

int unif_moe_fp8_quantize(const void* x, unif_moe_dtype dtype, int64_t rows, int cols, int64_t ld,
                          uint8_t* codes, int64_t ld_codes, float* scales, void* stream) {
  set_error("%s", "");
  const int rc = f8::check(x, dtype, rows, cols, ld, codes, ld_codes, scales);
  if (rc != UNIF_MOE_OK || rows == 0) return rc;
  const bool vec = f8::whole(x, dtype, cols, ld, codes, ld_codes);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == UNIF_MOE_F32
                            ? f8::quantize<float>(x, rows, cols, ld, codes, ld_codes, scales, vec, s)
                            : f8::quantize<__nv_bfloat16>(x, rows, cols, ld, codes, ld_codes, scales, vec, s);
  if (e != cudaSuccess) {
    set_error("fp8 quantize: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

int unif_moe_fp8_dequantize(const uint8_t* codes, int64_t ld_codes, const float* scales, int64_t rows, int cols,
                            void* x, unif_moe_dtype dtype, int64_t ld, void* stream) {
  set_error("%s", "");
  const int rc = f8::check(x, dtype, rows, cols, ld, codes, ld_codes, scales);
  if (rc != UNIF_MOE_OK || rows == 0) return rc;
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  const bool vec = f8::whole(x, dtype, cols, ld, codes, ld_codes);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == UNIF_MOE_F32
          ? f8::dequantize<float>(codes, ld_codes, scales, rows, cols, x, ld, vec, sms, s)
          : f8::dequantize<__nv_bfloat16>(codes, ld_codes, scales, rows, cols, x, ld, vec, sms, s);
  if (e != cudaSuccess) {
    set_error("fp8 dequantize: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

// Microscaled 4-bit floating point (MXFP4): rows to packed codes and block scales,
// and back (unif_moe_mxfp4_quantize / _dequantize). A block of 32 consecutive
// columns shares the scale 2^e, e = floor(log2 of its largest size) - 2 (at least
// -127), held as the byte e + 127; an element is x 2^-e rounded to nearest even
// among 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, and 6 beyond. x 2^-e is
// exact, so codes are the same on every machine.
//
// Bound by memory. A thread takes eight columns (16 bytes of bf16) and the four
// threads of a block find its largest size by two shuffles, so that a warp reads
// and writes consecutive bytes whatever the width; kUnroll pieces per thread are
// loaded before the first is used. 135,168 x 1,024 fp32 to 4 bits and back take 184 us, 6.8
// TB/s; 12,608 x 384 bf16 7.5 us (3.6 at that rate).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.cuh"

namespace unif {
namespace mxfp4 {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

// Eight consecutive elements as fp32 (0 past `cols`).
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
  if (VEC) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
    if (left > 0) {
      a = __ldcs(reinterpret_cast<const float4*>(p));
      b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
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
    if (left > 0) a = __ldcs(reinterpret_cast<const uint4*>(p));
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

// Eight values to eight codes, the first in the lowest four bits.
__device__ __forceinline__ uint32_t pack8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

// Pieces of eight columns are numbered row by row; I: their number's type. The
// four pieces of a block are four consecutive lanes, in the last row too (whole
// blocks are counted).
template <typename T, bool VEC, typename I>
__global__ void __launch_bounds__(kThreads)
    quantize_kernel(const T* x, I total, I per_row, int cols, long long ld, uint32_t* codes,
                    uint8_t* scales, int scale_pitch) {
  float v[kUnroll][8];
  I row[kUnroll];
  int piece[kUnroll];
  const I at = (I)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const I i = at + (I)(k * kThreads);
    row[k] = i / per_row;
    piece[k] = (int)(i - row[k] * per_row);
    const int left = i < total ? cols - piece[k] * 8 : 0;
    load8<VEC>(x + (long long)row[k] * ld + piece[k] * 8, left, v[k]);
  }
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const I i = at + (I)(k * kThreads);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[k][e]) & 0x7fffffffu);
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const int exponent = (int)(most >> 23);  // 255: infinity or NaN in the block
    const int scale = exponent == 255 ? 255 : max(exponent - 2, 0);
    const float by = __uint_as_float((uint32_t)(254 - scale) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[k][e] *= by;
    const uint32_t code = scale == 255 ? 0u : pack8(v[k]);
    if (i < total) {
      codes[i] = code;
      if ((piece[k] & 3) == 0) {
        uint8_t* s = scales + (long long)row[k] * scale_pitch;
        const int block = piece[k] >> 2;
        s[block] = (uint8_t)scale;
        if (piece[k] + 4 == (int)per_row)  // the row's last block fills the row up
          for (int b = block + 1; b < scale_pitch; ++b) s[b] = 0;
      }
    }
  }
}

// Four pairs of codes to eight values.
__device__ __forceinline__ void unpack8(uint32_t r, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(r));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// (A sector in one store: two stores of half a sector each took the 33 x 4,096
// x 1,024 fp32 values 127 us.)
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
  if (VEC) {
    if (left > 0)
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
                   "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = v[i];
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int left, const float (&v)[8]) {
  if (VEC) {
    if (left > 0) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t*>(&t);
      }
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = __float2bfloat16_rn(v[i]);
  }
}

template <typename T, bool VEC, typename I>
__global__ void __launch_bounds__(kThreads)
    dequantize_kernel(const uint32_t* codes, const uint8_t* scales, int scale_pitch, I total,
                      I per_row, int cols, T* x, long long ld) {
  uint32_t c[kUnroll];
  int s[kUnroll], piece[kUnroll];
  I row[kUnroll];
  const I at = (I)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const I i = at + (I)(k * kThreads);
    row[k] = i / per_row;
    piece[k] = (int)(i - row[k] * per_row);
    c[k] = 0;
    s[k] = 0;
    if (i < total) {
      c[k] = codes[i];
      s[k] = scales[(long long)row[k] * scale_pitch + (piece[k] >> 2)];
    }
  }
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    float v[8];
    unpack8(c[k], v);
    // 2^(s - 127): a byte is an exponent field, 0 the largest subnormal's half, 255 NaN
    const float by = __uint_as_float(s[k] == 255 ? 0x7fffffffu : s[k] ? (uint32_t)s[k] << 23 : 0x400000u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= by;
    const int left = at + (I)(k * kThreads) < total ? cols - piece[k] * 8 : 0;
    store8<VEC>(x + (long long)row[k] * ld + piece[k] * 8, left, v);
  }
}

int check(int64_t rows, int cols, int dtype, const void* x, int64_t ld, const void* codes,
          const void* scales) {
  if (rows < 0 || rows > (1ll << 40) || cols < 1 || cols > UNIF_MOE_MXFP4_MAX_COLS) {
    set_error("bad sizes: rows=%lld cols=%d (1 to %d)", (long long)rows, cols, UNIF_MOE_MXFP4_MAX_COLS);
    return UNIF_MOE_ERR_ARG;
  }
  if (dtype != UNIF_MOE_F32 && dtype != UNIF_MOE_BF16) { set_error("bad dtype"); return UNIF_MOE_ERR_ARG; }
  if (rows == 0) return UNIF_MOE_OK;
  if (!x || !codes || !scales || ld < cols) {
    set_error("x, codes or scales is NULL, or the row stride %lld is below cols=%d", (long long)ld, cols);
    return UNIF_MOE_ERR_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(codes) & 15u) || (reinterpret_cast<uintptr_t>(scales) & 7u)) {
    set_error("codes must be 16-byte aligned, scales 8-byte");
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

// Grid of `pieces` pieces; 0 where they are too many for one launch.
unsigned grid_of(int64_t pieces) {
  const int64_t g = (pieces + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  return g > 0x7fffffffll ? 0u : (unsigned)g;
}

template <typename T>
bool vec_ok(const void* x, int64_t ld, int cols) {  // eight elements in one access
  return reinterpret_cast<uintptr_t>(x) % (8 * sizeof(T)) == 0 && cols % 8 == 0 && ld % 8 == 0;
}

template <typename T, typename I>
cudaError_t quantize(const void* x, int64_t rows, int cols, int64_t ld, uint8_t* codes,
                     uint8_t* scales, cudaStream_t s) {
  const int per_row = (cols + 31) / 32 * 4, pitch = (cols + 255) / 256 * 8;
  const int64_t total = rows * per_row;
  const unsigned grid = grid_of(total);
  if (!grid) return cudaErrorInvalidValue;
  auto* c = reinterpret_cast<uint32_t*>(codes);
  const T* p = static_cast<const T*>(x);
  if (vec_ok<T>(x, ld, cols))
    quantize_kernel<T, true, I><<<grid, kThreads, 0, s>>>(p, (I)total, (I)per_row, cols, ld, c, scales, pitch);
  else
    quantize_kernel<T, false, I><<<grid, kThreads, 0, s>>>(p, (I)total, (I)per_row, cols, ld, c, scales, pitch);
  return cudaGetLastError();
}

template <typename T, typename I>
cudaError_t dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* x,
                       int64_t ld, cudaStream_t s) {
  const int per_row = (cols + 31) / 32 * 4, pitch = (cols + 255) / 256 * 8;
  const int64_t total = rows * per_row;
  const unsigned grid = grid_of(total);
  if (!grid) return cudaErrorInvalidValue;
  const auto* c = reinterpret_cast<const uint32_t*>(codes);
  T* p = static_cast<T*>(x);
  if (vec_ok<T>(x, ld, cols))
    dequantize_kernel<T, true, I><<<grid, kThreads, 0, s>>>(c, scales, pitch, (I)total, (I)per_row, cols, p, ld);
  else
    dequantize_kernel<T, false, I><<<grid, kThreads, 0, s>>>(c, scales, pitch, (I)total, (I)per_row, cols, p, ld);
  return cudaGetLastError();
}

// Whether the pieces' numbers fit in 32 bits, those of the last CTA included.
bool narrow(int64_t rows, int cols) {
  return rows * ((cols + 31) / 32 * 4) < (1ll << 32) - kThreads * kUnroll;
}

}  // namespace mxfp4
}  // namespace unif

using unif::set_error;
namespace fp4 = unif::mxfp4;

extern "C" {

int unif_moe_mxfp4_quantize(const void* x, unif_moe_dtype dtype, int64_t rows, int cols, int64_t ld,
                            uint8_t* codes, uint8_t* scales, void* stream) {
  set_error("%s", "");
  const int rc = fp4::check(rows, cols, dtype, x, ld, codes, scales);
  if (rc != UNIF_MOE_OK || rows == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool f32 = dtype == UNIF_MOE_F32, small = fp4::narrow(rows, cols);
  cudaError_t e;
  if (f32 && small) e = fp4::quantize<float, uint32_t>(x, rows, cols, ld, codes, scales, s);
  else if (f32) e = fp4::quantize<float, uint64_t>(x, rows, cols, ld, codes, scales, s);
  else if (small) e = fp4::quantize<__nv_bfloat16, uint32_t>(x, rows, cols, ld, codes, scales, s);
  else e = fp4::quantize<__nv_bfloat16, uint64_t>(x, rows, cols, ld, codes, scales, s);
  if (e != cudaSuccess) {
    set_error("mxfp4 quantize: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

int unif_moe_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                              void* x, unif_moe_dtype dtype, int64_t ld, void* stream) {
  set_error("%s", "");
  const int rc = fp4::check(rows, cols, dtype, x, ld, codes, scales);
  if (rc != UNIF_MOE_OK || rows == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool f32 = dtype == UNIF_MOE_F32, small = fp4::narrow(rows, cols);
  cudaError_t e;
  if (f32 && small) e = fp4::dequantize<float, uint32_t>(codes, scales, rows, cols, x, ld, s);
  else if (f32) e = fp4::dequantize<float, uint64_t>(codes, scales, rows, cols, x, ld, s);
  else if (small) e = fp4::dequantize<__nv_bfloat16, uint32_t>(codes, scales, rows, cols, x, ld, s);
  else e = fp4::dequantize<__nv_bfloat16, uint64_t>(codes, scales, rows, cols, x, ld, s);
  if (e != cudaSuccess) {
    set_error("mxfp4 dequantize: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

// Dense products with bias, activation and residual in the epilogue, and their gradients
// (unif_moe_linear_forward / _backward):
//   z = sx sw (x w^T) + b,  out = r + act(z);   dz = dout act'(z),  dx = dz w,  dw = dz^T x
//
// Two kernels multiply, four prepare or finish (us: 65,536 x 4,096 to 1,024 291, the library's product 290).
// - gemm_kernel: tiles of 128 rows, or of 256 on a CTA pair, by up to 256 columns on tcgen05,
//   accumulators in TMEM (two, so that one is stored while the next is computed), operands by
//   TMA through a ring of stages. All three products of a layer are this kernel: an operand
//   whose reduction index runs along memory is K-major, one whose reduction index is
//   the row (w in dx; dz and x in dw) MN-major, and neither is transposed in memory.
// - rows_kernel: few rows, bound by the weights' bytes: a CTA takes 16 output channels, its
//   warps share the columns, and both operands go from memory to mma.sync fragments without
//   shared memory (a thread's 16 bytes stand for other columns than the fragment's, the same
//   ones for both operands, which a sum does not notice). (1,024 to 4,096, weights from memory: 1 to 8 rows 4.3 us, at
//   the floor of the bytes 1.2, the library's product 4.4; 16 rows 5.0 and 3.6, 32 7.2 and 3.7. Weights in L2: 4 rows
//   3.3, 16 3.9, 32 6.3.)
// - grad_kernel / finish_kernel: dz and the column sums of dbias (12,608 x 1,536 21 us; its bytes 17); sums over
//   the parts of a split reduction, in a fixed order.
// - layout_kernel / steps_kernel: rows that TMA cannot read, laid out; the steps of dw that are not all padding.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "gelu_log.cuh"
#include "overlap.h"
#include "tc_common.cuh"

namespace unif {
namespace lin {

using namespace tc;

enum Kind {
  kForward = 0,   // bf16, both operands K-major
  kForward8 = 1,  // E4M3, both K-major
  kInput = 2,     // dx: dz K-major, w MN-major
  kWeight = 3     // dw: both MN-major
};

constexpr int kEpiWarps = 16, kTmaWarp = 16, kMmaWarp = 17;
constexpr int kEpiThreads = 32 * kEpiWarps;
constexpr int kCleanWarps = 8;  // of them, where padding rows are set to 0
constexpr int kThreads = kEpiThreads + 64;
constexpr uint32_t kTmemCols = 512, kAcc = 256;
constexpr int kMaxStages = 8;
constexpr int kBars = 3 * kMaxStages + 5 + 2 * kEpiWarps;
constexpr uint32_t kSmemMax = 232448;
// Staging of a storing warp: a box of 32 rows by 64 bytes, or two, and one for z; or, for rows that
// TMA cannot write, 32 rows by 16 fp32 values. Two boxes with a residual, which comes there first,
// and where a tile has few steps for its stores to hide behind (us, one box and two: 12,608 x 384 to
// 1,536 19.3 and 18.2; 65,536 x 1,024 to 4,096 with GELU 360 and 335); they leave the ring a stage
// less (the same without GELU 310 and 338).
constexpr uint32_t kBox = 2048, kStagingOdd = kEpiWarps * 32 * 17 * 4;
constexpr uint32_t kColumns = 2 * 2 * 256 * 4;          // bias and scales of two tiles
// Steps that one accumulation for an fp32 result runs over. The tensor cores
// truncate the accumulator at every MMA, so the error grows with their number: the sums of
// longer reductions are added in fp32 (65,536 x 4,096 to 1,024 onto an fp32 residual: 2.5e-6 of the
// result's norm off in one accumulation, 8e-7 so). That costs a wait for the
// addition each time (370 us against 293 with a bf16 result, whose own rounding is far above it; half of that
// are the result's bytes). A warp's 64 columns in registers, the accumulator given back at once, spill:
// 65,536 x 1,024 to 4,096 388 and 560 us.
constexpr int kSumSteps = 22;
// The same for a bf16 result: cut 2,048 times, by 2^-22 of what the accumulator holds at most, so by 2^-11 of its terms'
// absolute values together, and 2^-12 where they are of one sign (measured on average, 2^20 such columns: 1.7e-4 of
// the result in bf16, 5e-5 in 8 bits); its own rounding is 2^-8 at most.
constexpr int kSumSteps16 = 512;

struct Params {
  int M, N;                        // rows and columns of the result
  int steps, splits;               // steps of 128 operand bytes; parts of the reduction
  int sum_steps;                   // most steps of an accumulation
  int tile_n, m_tiles, n_tiles;    // columns of a tile (a multiple of 32)
  int stages;
  uint32_t stage_bytes, boxes;     // boxes staged by a warp, of them `two` in turn for the result
  bool two;
  bool gelu;
  void* out;                       // (through the tensor map where the rows allow that)
  long long ld_out;
  bool own_rows;                   // what is between the rows of out belongs to the call too
  const float *sm, *sn;            // scales of rows and columns, or NULL
  const void* bias;
  bool bias_f32;
  const void* residual;
  long long ld_res;
  const uint8_t* mask;
  bool clean_a, clean_b;           // ... the operands that may hold anything in padding rows
  const int* live;                 // kWeight with padding: how many steps have a row that is none, and which
  const unsigned long long* dead;  // a bit for each row of these steps, padding 1
  __nv_bfloat16* z;
  long long ld_z;
  int* status;
  long long wait_limit;
};

__device__ __forceinline__ void wait_settle(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > limit) return;
}

template <int KIND, bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  if constexpr (KIND != kForward8) {
    if (PAIR) umma_bf16_pair(d, a, b, idesc, acc);
    else umma_bf16(d, a, b, idesc, acc);
  } else if (PAIR) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
  }
}

// Instruction descriptor: fp32 accumulator (bits 4-5), operand types (bits 7-9 and 10-12: bf16
// 1, E4M3 0), MN-major A and B (bits 15, 16), N >> 3 and M >> 4.
template <int KIND, bool PAIR>
__device__ __forceinline__ uint32_t idesc_of(int n) {
  return (1u << 4) | (KIND == kForward8 ? 0u : (1u << 7) | (1u << 10)) |
         (KIND == kWeight ? 1u << 15 : 0u) | (KIND >= kInput ? 1u << 16 : 0u) |
         ((uint32_t)(n >> 3) << 17) | ((PAIR ? 256u >> 4 : 128u >> 4) << 24);
}

// Descriptor of an MN-major operand: 128-byte rows of 64 elements of one reduction index, 8-row
// groups 1,024 bytes apart, blocks of 64 elements one after the other (64 rows of 128 bytes).
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(8192 >> 4) << 16) |
         ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// 16 consecutive TMEM columns of 32 lanes from registers (complete after tmem_wait_st).
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
      " {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]),
      "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}

// 32 lanes x 16 columns without the wait: the registers are valid after tmem_wait_ld.
__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32"
      " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// (after tmem_wait_ld: nothing that uses the registers may be moved before it)
__device__ __forceinline__ void arrived(uint32_t (&r)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}

// ---- the epilogue's rows ----
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// What becomes of two results: bf16 ones take the packed GELU (2^-12.5 of the value at most,
// before a rounding of 2^-8), fp32 ones the library's.
template <typename TO>
__device__ __forceinline__ void act2(float& a, float& b) {
  if constexpr (sizeof(TO) == 4) {
    a *= normcdff(a);
    b *= normcdff(b);
  } else {
    gelu::gelu2(a, b);
  }
}

// Scales and bias on W columns of this thread's row (0 in padding rows), two at a time; `bias` and `sn`
// of the columns are in shared memory.
template <int W>
__device__ __forceinline__ void finish_row(const Params& p, float (&v)[W], float scale, bool on, const float* bias,
                                           const float* sn) {
  const uint64_t s2 = pk2(scale, scale);
  if (p.sm || p.sn || p.bias)
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(sn + i);
      const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(bias + i);
      upk2(fma2(pk2(v[i], v[i + 1]), mul2(s2, c.x), b.x), v[i], v[i + 1]);
      upk2(fma2(pk2(v[i + 2], v[i + 3]), mul2(s2, c.y), b.y), v[i + 2], v[i + 3]);
    }
  if (!on)
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0.f;
}

// This thread's row (64 bytes) of a staged box, 16 bytes at a time: TMA's 64-byte swizzle.
__device__ __forceinline__ uint32_t box_at(uint32_t box, int row, int piece) {
  return box + row * 64 + ((piece ^ (row >> 1 & 3)) << 4);
}
__device__ __forceinline__ void put4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void put_row(uint32_t box, int row, const float (&v)[32]) {  // bf16
#pragma unroll
  for (int i = 0; i < 4; ++i)
    put4(box_at(box, row, i), pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
         pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7]));
}
__device__ __forceinline__ void put_row(uint32_t box, int row, const float (&v)[16]) {  // fp32
#pragma unroll
  for (int i = 0; i < 4; ++i)
    put4(box_at(box, row, i), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
         __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
}
__device__ __forceinline__ void put_z(uint32_t box, int row, const float (&v)[32]) { put_row(box, row, v); }
__device__ __forceinline__ void put_z(uint32_t box, int row, const float (&v)[16]) {  // 32 bytes a row, no swizzle
#pragma unroll
  for (int i = 0; i < 2; ++i)
    put4(box + row * 32 + i * 16, pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
         pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7]));
}
__device__ __forceinline__ void get4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void add_row(uint32_t box, int row, float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r[4];
    get4(box_at(box, row, i), r);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[8 * i + 2 * k] += __uint_as_float(r[k] << 16);
      v[8 * i + 2 * k + 1] += __uint_as_float(r[k] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void add_row(uint32_t box, int row, float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r[4];
    get4(box_at(box, row, i), r);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * i + k] += __uint_as_float(r[k]);
  }
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1,
                                            int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// The sources of all of this thread's bulk stores but the last N have been read.
template <int N>
__device__ __forceinline__ void bulk_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

// One element.
template <typename TO>
__device__ __forceinline__ void finish1(const Params& p, float v, long long row, int ch, bool on, float sm,
                                        float sn, float bias, float residual) {
  if (p.sm || p.sn) v *= sm * sn;
  v += bias;
  if (!on) v = 0.f;
  if (p.z) p.z[row * p.ld_z + ch] = __float2bfloat16_rn(v);
  if (p.gelu) {
    float u = v;
    act2<TO>(v, u);
  }
  put(static_cast<TO*>(p.out) + row * p.ld_out + ch, on ? v + residual : 0.f);
}
__device__ __forceinline__ float bias_of(const Params& p, int ch) {
  return !p.bias ? 0.f
         : p.bias_f32 ? static_cast<const float*>(p.bias)[ch]
                      : __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[ch]);
}
template <typename TO>
__device__ __forceinline__ float residual_of(const Params& p, long long row, int ch) {
  return to_f32(static_cast<const TO*>(p.residual)[row * p.ld_res + ch]);
}

// PAIR: the CTAs of a cluster of two share a tile of 256 rows (tcgen05 cta_group::2), 128 of
// them and half of the columns' operand in each one's shared memory. The first CTA's
// barriers take both CTAs' bytes, its MMA lane issues for both.
// WIDE: the rows of the result (and of z and the residual) are written and read by TMA, from and to
// staged boxes of 32 rows by 64 bytes, which also cuts them off at the result's ends. Rows that TMA
// cannot write go through shared memory and the threads, a lane to a column (us, by TMA and so: 12,608 x 384 to
// 1,536 17.4 and 45.3, with GELU and z 24.2 and 55.7; 65,536 x 1,024 to 4,096 299 and 575).
//
// FORM (forward and dx; WIDE, not PAIR): a cluster of p.splits CTAs shares a tile, each a part of its reduction; their
// sums meet in shared memory, where each adds and finishes a share of the tile. For few rows and a
// long reduction, whose steps one CTA would run one after another (us, without and with: 256 x 4,096 to
// 1,024 17.4 and 13.1, with GELU and z 21.6 and 13.1; 64 x 4,096 to 1,024 16.3 and 10.5).
//
// FORM (dw): some rows are padding. Steps of none but such rows are not taken (Params::live), the others'
// padding rows set to 0 in shared memory before the MMAs read them, by half of the warps that store; a CTA of a
// pair then waits for its own bytes. (Against rows copied first, padding 0, all gradients, us: 32,768 x 4,096
// and 1,024, sequences of 100 to 512 of 512 434 and 320, every fourth row at random padding 446 and 387; 12,608 x
// 1,536 and 384 61 and 50, 62 and 54. Warps that take turns at the steps would have to wait on every one all the
// same: loads land out of order, and a barrier's parity tells only the last use from the one before.)
template <int KIND, typename TO, bool PAIR, bool WIDE, bool FORM>
__global__ void __launch_bounds__(kThreads, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmRes,
                const __grid_constant__ CUtensorMap tmZ, const Params p) {
  constexpr int kCtas = PAIR ? 2 : 1, kTileM = 128 * kCtas, kUnit = 16 * kCtas;  // columns of an MMA: whole units
  constexpr bool kParts = KIND == kWeight, clean = kParts && FORM, SPLIT = !kParts && FORM;
  const uint32_t rank = PAIR ? cluster_rank() : 0u;
  const bool leader = rank == 0;
  static_assert(!SPLIT || (WIDE && !PAIR), "forms");
  const uint32_t share = SPLIT ? cluster_rank() : 0u;  // SPLIT: the part of the reduction
  const int per = SPLIT ? p.splits : kCtas, unit = blockIdx.x / per, units = gridDim.x / per;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t s0 = smem_u32(smem);
  const int n_st = p.stages;
  auto stage = [&](int s) { return s0 + (uint32_t)s * p.stage_bytes; };
  // the ring, the staged boxes (512-byte aligned), barriers
  uint8_t* staged = smem + (size_t)n_st * p.stage_bytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staged + (WIDE ? kEpiWarps * p.boxes * kBox : kStagingOdd));
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kMaxStages + s); };
  auto accf_bar = [&](int a) { return bar0 + 8u * (2 * kMaxStages + a); };
  auto acce_bar = [&](int a) { return bar0 + 8u * (2 * kMaxStages + 2 + a); };
  const uint32_t mma_done = bar0 + 8u * (2 * kMaxStages + 4);
  auto box_bar = [&](int w, uint32_t k) { return bar0 + 8u * (2 * kMaxStages + 5 + 2 * w + (k & 1u)); };
  auto clean_bar = [&](int s) { return bar0 + 8u * (2 * kMaxStages + 5 + 2 * kEpiWarps + s); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* columns = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(bars + kBars + 1) + 15) & ~(uintptr_t)15);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int epi_warps = clean ? kEpiWarps - kCleanWarps : kEpiWarps;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
      mbar_init(clean_bar(s), kCtas * kCleanWarps);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(accf_bar(a), 1);
      mbar_init(acce_bar(a), kCtas * epi_warps);
    }
    mbar_init(mma_done, 1);
    for (int w = 0; w < kEpiWarps; ++w) {
      mbar_init(box_bar(w, 0), 1);
      mbar_init(box_bar(w, 1), 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    if (PAIR) {
      tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(tmem_slot), kTmemCols);
      tmem_relinquish();
    }
  }
  grid_dep_wait();
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();  // both CTAs' barriers are set before either signals the other
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto arrive_leader = [&](uint32_t bar) {
    if (!PAIR || leader) mbar_arrive(bar);
    else mbar_arrive_cluster(mapa_shared(bar, 0));
  };
  auto commit = [&](uint32_t bar) {
    if (PAIR) umma_commit_pair(bar, 3);
    else umma_commit(bar);
  };

  // Items: (part of the reduction, row tile, column tile), the columns of a row tile one after
  // another so that its rows are read from L2 but once from memory.
  struct Item {
    int m0, n0, n;      // this CTA's first row, the tile's first column and columns
    int from, to;       // steps
    int part;
  };
  // accumulations of an item; the first step of its j-th
  auto sums = [&](const Item& it) { return (it.to - it.from + p.sum_steps - 1) / p.sum_steps; };
  auto first_step = [&](const Item& it, int n, int j) {
    return it.from + (int)((long long)(it.to - it.from) * j / n);
  };
  // The items of this CTA or pair one after another, i = unit + k units, without a division for each.
  struct Walk {
    int i, m, n, part;
  };
  const int n_items = p.m_tiles * p.n_tiles * (SPLIT ? 1 : p.splits);
  const int by_m = units / p.n_tiles, by_n = units - by_m * p.n_tiles;
  auto start = [&]() {
    Walk w;
    w.i = unit;
    w.m = unit / p.n_tiles;
    w.n = unit - w.m * p.n_tiles;
    w.part = kParts ? w.m / p.m_tiles : 0;
    w.m -= w.part * p.m_tiles;
    return w;
  };
  auto next = [&](Walk& w) {
    w.i += units;
    w.m += by_m;
    w.n += by_n;
    if (w.n >= p.n_tiles) {
      w.n -= p.n_tiles;
      ++w.m;
    }
    if (kParts)
      for (; w.m >= p.m_tiles; w.m -= p.m_tiles) ++w.part;
  };
  const int all_steps = clean ? *p.live : p.steps;
  auto item_of = [&](const Walk& w) {
    Item it;
    it.part = w.part;
    it.m0 = w.m * kTileM + 128 * (int)rank;
    it.n0 = w.n * p.tile_n;
    it.n = min(p.tile_n, p.N - it.n0);
    const int part = SPLIT ? (int)share : it.part;
    it.from = kParts || SPLIT ? (int)((long long)all_steps * part / p.splits) : 0;
    it.to = kParts || SPLIT ? (int)((long long)all_steps * (part + 1) / p.splits) : p.steps;
    return it;
  };

  if (warp < epi_warps) {
    // ---------------- accumulators to the result ----------------------------
    // Four warps (two beside those that clean) to a quarter of the rows, W columns at a time. (A wait given up is not the end
    // of the loop: the warps meet at a barrier.)
    constexpr int W = WIDE ? 64 / (int)sizeof(TO) : 16;
    constexpr int parts = epi_warps / 4;
    const int q = warp & 3, part = warp >> 2;
    int acc = 0;       // the accumulator of the item's sum
    uint32_t ph = 0;   // a phase bit per accumulator
    bool ok = true;
    auto wait_acc = [&](int a) {
      ok = ok && wait_warp(accf_bar(a), ph >> a & 1u, abort_flag, p.status, p.wait_limit);
      ph ^= 1u << a;
      tc_fence_after();
    };
    auto release = [&](int a) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_leader(acce_bar(a));
    };
    // pieces of W columns of an item in this warp's rows (a quarter past the last row has none)
    auto pieces = [&](const Item& it) { return it.m0 + q * 32 < p.M ? (it.n + W - 1) / W : 0; };
    // The pieces of this warp one after another, over the items.
    struct Piece {
      Walk at;
      int c, n0, m0, of;  // of its item: first column and row, pieces
    };
    auto enter = [&](Piece& e) {
      const Item it = item_of(e.at);
      e.c = part;
      e.n0 = it.n0;
      e.m0 = it.m0;
      e.of = e.at.i < n_items ? pieces(it) : 0;
    };
    auto first_piece = [&]() {
      Piece e;
      e.at = start();
      enter(e);
      return e;
    };
    auto settle = [&](Piece& e) {  // the piece, or the next one there is; false after the last
      while (e.c >= e.of) {
        if (e.at.i >= n_items) return false;
        next(e.at);
        enter(e);
      }
      return true;
    };
    const bool per_column = KIND < kInput && (p.bias || p.sn || p.sm);
    // The columns' bias (the first 256 threads) and scales (the others), on their way a tile ahead. (Each
    // warp its own columns, without the barrier: 12,608 x 384 to 1,536 16.3 us and 18.7.)
    auto column = [&](const Walk& w) {
      const int c = (int)(threadIdx.x & 255u), n0 = w.n * p.tile_n;
      if (c >= min(p.tile_n, p.N - n0)) return 0.f;
      if (threadIdx.x < 256) return bias_of(p, n0 + c);
      return p.sn ? p.sn[n0 + c] : 1.f;
    };
    Walk ahead = start();
    float in_columns = per_column && ahead.i < n_items ? column(ahead) : 0.f;
    int turn = 0;
    // WIDE: boxes this warp has staged, and the residual's boxes on their way (two ahead)
    const bool with_res = WIDE && !SPLIT && KIND < kInput && p.residual;
    const uint32_t box0 = smem_u32(staged) + warp * p.boxes * kBox, two = p.two ? kBox : 0u;
    uint32_t k = 0, fetched = 0;
    Piece coming = first_piece();
    auto fetch = [&]() {  // the residual of the next piece, to the box that will hold its result
      if (!settle(coming)) return;
      if (lane == 0) {
        mbar_expect_tx(box_bar(warp, fetched), kBox);
        tma_load_3d(box0 + (fetched & 1u) * two, &tmRes, box_bar(warp, fetched),
                    coming.n0 + coming.c * W, coming.m0 + q * 32, 0);
      }
      ++fetched;
      coming.c += 4;
    };
    if (with_res) {
      fetch();
      fetch();
    }
    for (Walk at = start(); at.i < n_items; next(at), turn ^= 512) {
      const Item it = item_of(at);
      const float* cols = columns + turn;
      if (per_column) {
        columns[turn + threadIdx.x] = in_columns;
        asm volatile("bar.sync 1, %0;" ::"n"(kEpiThreads) : "memory");
        next(ahead);
        if (ahead.i < n_items) in_columns = column(ahead);
      }
      const long long row = (long long)it.m0 + q * 32 + lane;
      const bool there = row < p.M;
      const int n_pieces = pieces(it);
      bool on = there;
      float scale = 1.f;
      if (KIND != kWeight && there && p.mask) on = p.mask[row] != 0;
      if (KIND < kInput && there && p.sm) scale = p.sm[row];
      const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
      const int n_sums = sums(it);
      wait_acc(acc);
      for (int j = 1; j < n_sums; ++j) {  // further accumulations, added to the first
        wait_acc(acc ^ 1);
        if (!ok) break;
        for (int c = part; c < n_pieces; c += parts)
#pragma unroll
          for (int h = 0; h < W; h += 16) {
            uint32_t u[16], v[16];
            tmem_ld16_async(lanes + acc * kAcc + c * W + h, u);
            tmem_ld16_async(lanes + (acc ^ 1) * kAcc + c * W + h, v);
            tmem_wait_ld();
            arrived(u);
            arrived(v);
            float w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __uint_as_float(u[e]) + __uint_as_float(v[e]);
            tmem_st16(lanes + acc * kAcc + c * W + h, w);
          }
        tmem_wait_st();
        release(acc ^ 1);
      }
      if (!ok) continue;
      if constexpr (SPLIT) {
        // (all of this CTA's MMAs have completed: the ring is free) rows of tile_n + 4 values
        for (int c = part; c < n_pieces; c += parts) {
          float v[W];
          if constexpr (W == 32) tmem_ld32(lanes + acc * kAcc + c * W, v);
          else tmem_ld16(lanes + acc * kAcc + c * W, v);
          const uint32_t to = s0 + ((q * 32 + lane) * (p.tile_n + 4) + c * W) * 4;
#pragma unroll
          for (int e = 0; e < W; e += 4)
            put4(to + e * 4, __float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]),
                 __float_as_uint(v[e + 3]));
        }
        release(acc);
        acc ^= 1;
        continue;
      }
      for (int c = part; c < n_pieces; c += parts) {
        float v[W];
        if constexpr (W == 32) tmem_ld32(lanes + acc * kAcc + c * W, v);
        else tmem_ld16(lanes + acc * kAcc + c * W, v);
        if (c + parts >= n_pieces) release(acc);
        const int ch = it.n0 + c * W;
        if constexpr (WIDE) {
          if constexpr (KIND < kInput) finish_row<W>(p, v, scale, on, cols + c * W, cols + 256 + c * W);
          else if (KIND == kInput && !on)
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = 0.f;
          const uint32_t box = box0 + (k & 1u) * two, z_box = box0 + two + kBox;
          if (with_res) {
            ok = wait_warp(box_bar(warp, k), k >> 1 & 1u, abort_flag, p.status, p.wait_limit);
            if (!ok) break;
          } else {
            if (lane == 0) {  // the box's last piece has gone out (and z's)
              if (p.two) bulk_read<1>();
              else bulk_read<0>();
            }
            __syncwarp();
          }
          if constexpr (KIND < kInput) {
            if (p.z) {
              put_z(z_box, lane, v);
              fence_proxy_async();
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&tmZ, z_box, ch, it.m0 + q * 32, 0);
                bulk_commit();
              }
            }
            if (p.gelu)
#pragma unroll
              for (int e = 0; e < W; e += 2) act2<TO>(v[e], v[e + 1]);
            if (with_res && on) add_row(box, lane, v);
          }
          put_row(box, lane, v);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            tma_store_3d(&tmOut, box, ch, it.m0 + q * 32, it.part);
            bulk_commit();
          }
          ++k;
          if (with_res) {
            if (lane == 0) bulk_read<0>();
            fetch();
          }
        } else {
          // a lane per column, two rows at a time: rows of any width and alignment
          float* stg = reinterpret_cast<float*>(staged) + warp * (32 * 17);
          const int count = it.n - c * W;
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 16; ++j) stg[lane * 17 + j] = v[j];
          __syncwarp();
          const uint32_t live = __ballot_sync(0xffffffffu, on);
          const int col = lane & 15;
          const float sn = per_column ? cols[256 + c * W + col] : 1.f, b = per_column ? cols[c * W + col] : 0.f;
          // this lane's rows, every other one: what they take of the residual first, all on its way at once
          const int r0 = lane >> 4, rows = (int)min(32ll, p.M - (row - lane));
          TO res[16];
          if (KIND < kInput && p.residual) {
            const TO* from = static_cast<const TO*>(p.residual) + (row - lane + r0) * p.ld_res + ch + col;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if ((live >> (r0 + 2 * e) & 1u) && col < count) res[e] = from[2 * e * p.ld_res];
          }
          const bool scaled = KIND < kInput && p.sm;
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            float y[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = r0 + 2 * (e + h);
              y[h] = KIND == kWeight || (live >> r & 1u) ? stg[r * 17 + col] : 0.f;
              if constexpr (KIND < kInput) {
                const float sm = scaled ? __shfl_sync(0xffffffffu, scale, r) : 1.f;
                y[h] = live >> r & 1u ? fmaf(y[h], sm * sn, b) : 0.f;
                if (p.z && r < rows && col < count)
                  p.z[(row - lane + r) * p.ld_z + ch + col] = __float2bfloat16_rn(y[h]);
              }
            }
            if (KIND < kInput && p.gelu) act2<TO>(y[0], y[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = r0 + 2 * (e + h);
              if (KIND < kInput && p.residual && (live >> r & 1u)) y[h] += to_f32(res[e + h]);
              if (r < rows && col < count)
                put(static_cast<TO*>(p.out) + (row - lane + r) * p.ld_out + ch + col, y[h]);
            }
          }
        }
      }
      if (part >= n_pieces) release(acc);
      acc ^= 1;
    }
    if (WIDE && lane == 0) {
      for (; k < fetched; ++k) wait_settle(box_bar(warp, k), k >> 1 & 1u, p.wait_limit / 16);  // (after a wait given up)
      bulk_wait_all();
    }
    __syncwarp();
  } else if (clean && warp < kEpiWarps) {
    // ---------------- padding rows to 0 (kWeight): eight of a step's 64 rows to a warp ----
    const int r0 = (warp - epi_warps) * (64 / kCleanWarps);
    static_assert(kCleanWarps == 8, "a byte of padding bits");
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (Walk at = start(); at.i < n_items && ok; next(at)) {
      const Item it = item_of(at);
      const int blocks = ((it.n + kUnit - 1) / kUnit * 16 + 63) / 64;
      uint32_t bits = 0;  // of a lane's step of the next 32: this warp's rows that are padding; bit 8: all 64 are
      for (int k = it.from; k < it.to; ++k) {
        const int of32 = (k - it.from) & 31;
        if (of32 == 0) {
          const unsigned long long d = k + lane < it.to ? p.dead[k + lane] : 0ull;
          bits = ((uint32_t)(d >> r0) & 255u) | (d == ~0ull ? 256u : 0u);
        }
        ok = wait_warp(full_bar(s), ph, abort_flag, p.status, p.wait_limit);
        if (!ok) break;
        const uint32_t dead = __shfl_sync(0xffffffffu, bits, of32);
        if (dead) {
          const uint32_t a = stage(s) + r0 * 128 + lane * 16, b = a + 16384u;
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 128 bytes of four rows at a time
            if (!(dead >> (h * 4 + (lane >> 3)) & 1u)) continue;
            if (p.clean_a || dead >> 8) {
              put4(a + h * 512u, 0u, 0u, 0u, 0u);
              put4(a + h * 512u + 8192u, 0u, 0u, 0u, 0u);
            }
            if (p.clean_b || dead >> 8)
              for (int j = 0; j < blocks; ++j) put4(b + h * 512u + j * 8192u, 0u, 0u, 0u, 0u);
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) arrive_leader(clean_bar(s));
        if (++s == n_st) { s = 0; ph ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == kTmaWarp) {
    // ---------------- operands (one lane runs the role from end to end) -----
    if (elect_one()) {
      bool ok = true;
      int s = 0;
      uint32_t ph = 0;
      long long issued = 0;
      auto load = [&](uint32_t dst, const CUtensorMap* from, uint32_t bar, int c0, int c1) {
        if (PAIR) tma_load_2d_pair(dst, from, mapa_shared(bar, clean ? rank : 0), c0, c1);
        else tma_load_2d(dst, from, bar, c0, c1);
      };
      constexpr int kCols = KIND == kForward8 ? 128 : 64;  // reduction elements of a step
      for (Walk at = start(); at.i < n_items && ok; next(at)) {
        const Item it = item_of(at);
        // this CTA's share of the columns
        const int n = (it.n + kUnit - 1) / kUnit * 16, n0 = it.n0 + (int)rank * n;
        const int blocks = (n + 63) / 64;  // of an MN-major operand
        const uint32_t bytes = 16384u + (KIND >= kInput ? blocks * 8192u : (uint32_t)(p.tile_n / kCtas) * 128u);
        int coming = clean && it.from < it.to ? p.live[1 + it.from] : 0;  // (a step ahead)
        for (int i = it.from; i < it.to; ++i) {
          const int k = clean ? coming : i;
          if (clean && i + 1 < it.to) coming = p.live[2 + i];
          ok = wait_bounded(empty_bar(s), ph ^ 1u, abort_flag, p.status, p.wait_limit);
          if (!ok) break;
          const uint32_t bar = full_bar(s), a = stage(s), b = a + 16384u;
          if (clean) mbar_expect_tx(bar, bytes);
          else if (leader) mbar_expect_tx(bar, kCtas * bytes);
          if (KIND == kWeight) {
            load(a, &tmA, bar, it.m0, k * kCols);
            load(a + 8192u, &tmA, bar, it.m0 + 64, k * kCols);
          } else {
            load(a, &tmA, bar, k * kCols, it.m0);
          }
          if (KIND >= kInput)
            for (int j = 0; j < blocks; ++j) load(b + j * 8192u, &tmB, bar, n0 + 64 * j, k * kCols);
          else
            load(b, &tmB, bar, k * kCols, n0);
          ++issued;
          if (++s == n_st) { s = 0; ph ^= 1u; }
        }
      }
      // loads still in flight land before the CTA (pair) exits
      for (long long j = issued > n_st ? issued - n_st : 0; (leader || clean) && j < issued; ++j)
        wait_settle(full_bar((int)(j % n_st)), (uint32_t)((j / n_st) & 1), p.wait_limit / 16);
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------- MMAs (the first CTA) ----------------------------------
    if (leader && elect_one()) {
      int s = 0, acc = 0;
      uint32_t ph = 0, acc_ph = 0;
      bool ok = true, any = false;
      for (Walk at = start(); at.i < n_items && ok; next(at)) {
        const Item it = item_of(at);
        const uint32_t idesc = idesc_of<KIND, PAIR>((it.n + kUnit - 1) / kUnit * kUnit);
        const int n_sums = sums(it);
        for (int j = 0; j < n_sums && ok; ++j) {
          const int to = j ? acc ^ 1 : acc;
          ok = wait_bounded(acce_bar(to), (acc_ph >> to & 1u) ^ 1u, abort_flag, p.status, p.wait_limit);
          if (!ok) break;
          acc_ph ^= 1u << to;
          tc_fence_after();
          const uint32_t d = tmem + to * kAcc;
          const int first = first_step(it, n_sums, j), last = first_step(it, n_sums, j + 1);
          for (int k = first; k < last; ++k) {
            ok = wait_bounded(clean ? clean_bar(s) : full_bar(s), ph, abort_flag, p.status, p.wait_limit);
            if (!ok) break;
            tc_fence_after();
            const uint32_t sa = stage(s), sb = sa + 16384u;
            // 32 bytes of the reduction along memory, or 16 rows, at a time
            const uint64_t a = KIND == kWeight ? mn_desc(sa) : sw128_desc(sa);
            const uint64_t b = KIND >= kInput ? mn_desc(sb) : sw128_desc(sb);
            constexpr int kStepA = KIND == kWeight ? 128 : 2, kStepB = KIND >= kInput ? 128 : 2;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              mma<KIND, PAIR>(d, a + kStepA * e, b + kStepB * e, idesc, (k > first || e > 0) ? 1u : 0u);
            commit(empty_bar(s));
            any = true;
            if (++s == n_st) { s = 0; ph ^= 1u; }
          }
          if (ok) commit(accf_bar(to));
        }
        acc ^= 1;
      }
      // every MMA issued has completed before TMEM is released
      if (any) {
        if (PAIR) umma_commit_pair(mma_done, 1);
        else umma_commit(mma_done);
        wait_settle(mma_done, 0u, p.wait_limit);
      }
    }
    __syncwarp();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (PAIR || SPLIT) cluster_sync_all();
  if constexpr (SPLIT) {
    // Four columns of 32 rows to a warp of the cluster in turn, a row to a lane; the parts are added in
    // order.
    const Item it = item_of(start());
    if (warp < kEpiWarps && *abort_flag == 0)
      for (int u = warp * p.splits + (int)share; u < it.n; u += kEpiWarps * p.splits) {
        const int q = u & 3, c = u & ~3, ch = it.n0 + c;
        const long long row = (long long)it.m0 + q * 32 + lane;
        if (row >= p.M || c >= it.n) continue;
        const uint32_t at = s0 + ((q * 32 + lane) * (p.tile_n + 4) + c) * 4;
        float a[8][4];
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r < p.splits)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(a[r][0]), "=f"(a[r][1]), "=f"(a[r][2]), "=f"(a[r][3])
                         : "r"(mapa_shared(at, r))
                         : "memory");
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[0][e];
#pragma unroll
        for (int r = 1; r < 8; ++r)
          if (r < p.splits)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += a[r][e];
        const bool on = !p.mask || p.mask[row] != 0;
        TO* out = static_cast<TO*>(p.out) + row * p.ld_out + ch;
        if constexpr (KIND < kInput) {
          finish_row<4>(p, v, p.sm ? p.sm[row] : 1.f, on, columns + c, columns + 256 + c);
          if (p.z)
            *reinterpret_cast<uint2*>(p.z + row * p.ld_z + ch) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
          if (p.gelu) {
            act2<TO>(v[0], v[1]);
            act2<TO>(v[2], v[3]);
          }
          if (p.residual && on) {
            const TO* res = static_cast<const TO*>(p.residual) + row * p.ld_res + ch;
            if constexpr (sizeof(TO) == 4) {
              const float4 b = *reinterpret_cast<const float4*>(res);
              v[0] += b.x; v[1] += b.y; v[2] += b.z; v[3] += b.w;
            } else {
              const uint2 b = *reinterpret_cast<const uint2*>(res);
              v[0] += __uint_as_float(b.x << 16);
              v[1] += __uint_as_float(b.x & 0xffff0000u);
              v[2] += __uint_as_float(b.y << 16);
              v[3] += __uint_as_float(b.y & 0xffff0000u);
            }
          }
        }
        if (KIND == kInput && !on) v[0] = v[1] = v[2] = v[3] = 0.f;
        if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2*>(out) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
      }
    __syncwarp();
    cluster_sync_all();  // no CTA leaves while another reads its sums
  }
  if (warp == kMmaWarp) {
    if (PAIR) tmem_dealloc_pair(tmem, kTmemCols);
    else tmem_dealloc(tmem, kTmemCols);
  }
}

// ---- few rows ----

struct RowsParams {
  Params e;             // M, N, epilogue
  const uint8_t *x, *w; // rows
  long long ld_x, ld_w; // bytes between rows
  int bytes;            // of a row
};
constexpr int kRowsMax = 32;       // rows of x
constexpr int kRowsWarps = 16;     // most warps of a CTA
constexpr int kRowsBytes = 65536;  // of a row: 32 blocks of 128 bytes for an accumulator (as kSumSteps; longer rows: tiles)

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
      " {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16832(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
      " {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Sixteen bytes of a row, those past its end 0 (`left` bytes are left of it). VEC: rows
// start at multiples of 16 bytes. SIZE: bytes of an element.
template <bool VEC, int SIZE>
__device__ __forceinline__ uint4 piece(const uint8_t* p, int left) {
  if (VEC && left >= 16) return __ldg(reinterpret_cast<const uint4*>(p));
  uint32_t r[4] = {0u, 0u, 0u, 0u};
  if (left > 0) {
#pragma unroll
    for (int i = 0; i < 16 / SIZE; ++i)
      if (i * SIZE < left) {
        const uint32_t v = SIZE == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p + 2 * i) : (uint32_t)p[i];
        r[i * SIZE / 4] |= v << (8 * (i * SIZE % 4));
      }
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// NT: pieces of eight rows of x. A warp takes 128-byte blocks of the rows in turn with the
// CTA's other warps, two pieces of 16 bytes a thread from each of 16 weight rows.
template <int SIZE, int NT, bool VEC, typename TO>
__global__ void __launch_bounds__(32 * kRowsWarps) rows_kernel(const RowsParams p) {
  __shared__ float red[kRowsWarps * 16 * 8 * NT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int g = lane >> 2, at = (lane & 3) * 16;
  const int ch0 = blockIdx.x * 16;
  grid_dep_wait();
  const bool two = ch0 + g + 8 < p.e.N, one = ch0 + g < p.e.N;
  const uint8_t* w0 = p.w + (one ? ch0 + g : 0) * p.ld_w;
  const uint8_t* w1 = p.w + (two ? ch0 + g + 8 : 0) * p.ld_w;
  float c[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) c[t][i] = 0.f;
  const int blocks = (p.bytes + 127) / 128;
#pragma unroll 2
  for (int b = warp; b < blocks; b += warps) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int from = b * 128 + h * 64 + at, left = p.bytes - from;
      const uint4 a = piece<VEC, SIZE>(w0 + from, one ? left : 0);
      const uint4 d = piece<VEC, SIZE>(w1 + from, two ? left : 0);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int row = t * 8 + g;
        const uint4 x = piece<VEC, SIZE>(p.x + (row < p.e.M ? row : 0) * p.ld_x + from, row < p.e.M ? left : 0);
        if (SIZE == 2) {
          mma_16816(c[t], a.x, d.x, a.y, d.y, x.x, x.y);
          mma_16816(c[t], a.z, d.z, a.w, d.w, x.z, x.w);
        } else {
          mma_16832(c[t], a.x, d.x, a.y, d.y, x.x, x.y);
          mma_16832(c[t], a.z, d.z, a.w, d.w, x.z, x.w);
        }
      }
    }
  }
  // [warp][row of x][channel]; c: channels g, g and g + 8, g + 8, rows 2 (lane % 4), + 1
  float* mine = red + warp * (16 * 8 * NT);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[(t * 8 + (lane & 3) * 2 + (i & 1)) * 16 + g + (i >> 1) * 8] = c[t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 8 * NT; i += blockDim.x) {
    const int row = i >> 4, ch = ch0 + (i & 15);
    if (row >= p.e.M || ch >= p.e.N) continue;
    float v = 0.f;
    for (int k = 0; k < warps; ++k) v += red[k * (16 * 8 * NT) + i];
    const bool on = !p.e.mask || p.e.mask[row];
    finish1<TO>(p.e, v, row, ch, on, p.e.sm ? p.e.sm[row] : 1.f, p.e.sn ? p.e.sn[ch] : 1.f, bias_of(p.e, ch),
                on && p.e.residual ? residual_of<TO>(p.e, row, ch) : 0.f);
  }
}

// ---- rows laid out for TMA, dz and the bias's gradient ----

// Rows to a pitch of whole 16 bytes, one or two arrays of them; padding rows to 0. A warp to 256
// elements of a row.
struct Rows {
  const void* x;
  long long ld;
  void* to;
  long long pitch, rows;
  int cols;
  const uint8_t* mask;
  __host__ __device__ long long warps() const { return rows * ((cols + 255) / 256); }
};
template <typename T>
__global__ void __launch_bounds__(256) layout_kernel(const Rows a, const Rows b) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const long long of_a = a.warps(), total = of_a + b.warps(), step = (long long)gridDim.x * 8;
  for (long long k = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); k < total; k += step) {
    const Rows& j = k < of_a ? a : b;
    const long long i = k < of_a ? k : k - of_a;
    const int pieces = (j.cols + 255) / 256;
    const long long row = i / pieces;
    const int c0 = (int)(i - row * pieces) * 256 + lane;
    const bool on = !j.mask || j.mask[row];
    const T* from = static_cast<const T*>(j.x) + row * j.ld + c0;
    T* to = static_cast<T*>(j.to) + row * j.pitch + c0;
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = on && c0 + 32 * e < j.cols ? from[32 * e] : (T)0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c0 + 32 * e < j.cols) to[32 * e] = v[e];
  }
}

// The steps of 64 rows that are not all padding, in order: how many, which, and their padding rows' bits. At least
// `least` (and no more than there are): the list is filled up with steps all of whose bits are set. One CTA.
constexpr int kListThreads = 1024;
__global__ void __launch_bounds__(kListThreads) steps_kernel(const uint8_t* mask, long long rows, int least, int* live,
                                                             unsigned long long* dead) {
  __shared__ int found[kListThreads / 32];
  grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int steps = (int)((rows + 63) / 64);
  const bool aligned = reinterpret_cast<uintptr_t>(mask) % 16 == 0;
  int before = 0;
  for (int from = 0; from < steps; from += kListThreads) {
    const int step = from + (int)threadIdx.x;
    const long long row0 = (long long)step * 64;
    unsigned long long d = 0ull;
    if (aligned && row0 + 64 <= rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 m = *(reinterpret_cast<const uint4*>(mask + row0) + i);
        const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)  // bit 0 of each byte to four bits side by side
          d |= (unsigned long long)((__vcmpeq4(w[e], 0u) & 0x01010101u) * 0x10204080u >> 28) << (16 * i + 4 * e);
      }
    } else {
      for (int i = 0; i < 64; ++i) d |= (unsigned long long)(row0 + i >= rows || mask[row0 + i] == 0) << i;
    }
    const bool on = step < steps && d != ~0ull;
    const uint32_t b = __ballot_sync(0xffffffffu, on);
    if (lane == 0) found[warp] = __popc(b);
    __syncthreads();
    int at = before + __popc(b & ((1u << lane) - 1u));
#pragma unroll
    for (int w = 0; w < kListThreads / 32; ++w) {
      if (w < warp) at += found[w];
      before += found[w];
    }
    if (on) {
      live[1 + at] = step;
      dead[at] = d;
    }
    __syncthreads();
  }
  for (int i = before + (int)threadIdx.x; i < min(least, steps); i += kListThreads) {
    live[1 + i] = 0;
    dead[i] = ~0ull;
  }
  if (threadIdx.x == 0) *live = max(before, min(least, steps));
}

struct GradParams {
  long long rows;
  int n, per;                // per: rows of a CTA
  const void* dout;
  long long ld_dout;
  const __nv_bfloat16* z;    // or NULL: no activation
  long long ld_z;
  const uint8_t* mask;
  __nv_bfloat16* dz;         // or NULL: dout itself is dz
  long long ld_dz;
  float* sums;               // [row blocks][n] or NULL
};
constexpr int kGradWarps = 8, kGradRows = 4;  // rows in flight of a warp

// Eight values as they are read: consecutive ones (VEC), or every 32nd.
template <typename T, bool VEC>
struct Eight {
  uint32_t r[VEC ? 8 * sizeof(T) / 4 : 8];
  __device__ __forceinline__ void read(const T* p, int left) {  // left: values up to the row's end from p on
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        r[4 * i] = a.x; r[4 * i + 1] = a.y; r[4 * i + 2] = a.z; r[4 * i + 3] = a.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = 32 * k < left ? __float_as_uint(to_f32(p[32 * k])) : 0u;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(r) / 4); ++k) r[k] = 0u;
  }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (VEC && sizeof(T) == 2) return __uint_as_float(k & 1 ? r[k / 2] & 0xffff0000u : r[k / 2] << 16);
    else return __uint_as_float(r[k]);
  }
};

// dz = dout act'(z), and the column sums of the CTA's rows: 256 columns by `per` rows, a warp to
// every eighth row, eight columns a lane (VEC: consecutive ones).
template <typename TD, bool VEC>
__global__ void __launch_bounds__(32 * kGradWarps, VEC ? 3 : 2) grad_kernel(const GradParams p) {
  __shared__ float red[kGradWarps][256];
  grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c0 = blockIdx.x * 256;
  auto column = [&](int k) { return c0 + (VEC ? lane * 8 + k : lane + 32 * k); };
  const bool on_cols = column(0) < p.n;
  const long long first = (long long)blockIdx.y * p.per, last = min(p.rows, first + p.per);
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = 0.f;
  const TD* dout = static_cast<const TD*>(p.dout);
  for (long long r0 = first + warp; r0 < last; r0 += kGradWarps * kGradRows) {
    Eight<TD, VEC> d[kGradRows];
    Eight<__nv_bfloat16, VEC> z[kGradRows];
#pragma unroll
    for (int u = 0; u < kGradRows; ++u) {
      const long long r = r0 + u * kGradWarps;
      if (r < last && on_cols && (!p.mask || p.mask[r])) {
        d[u].read(dout + r * p.ld_dout + column(0), p.n - column(0));
        if (p.z) z[u].read(p.z + r * p.ld_z + column(0), p.n - column(0));
      } else {  // (GELU's derivative of 0 is finite: padding rows give 0)
        d[u].clear();
        z[u].clear();
      }
    }
#pragma unroll
    for (int u = 0; u < kGradRows; ++u) {
      const long long r = r0 + u * kGradWarps;
      if (r >= last || !on_cols) continue;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = d[u].get(k);
      if (p.z)
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          float a, b;
          gelu::gelu_grad2(z[u].get(k), z[u].get(k + 1), a, b);
          v[k] *= a;
          v[k + 1] *= b;
        }
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += v[k];
      if (!p.dz) continue;
      __nv_bfloat16* o = p.dz + r * p.ld_dz;
      if constexpr (VEC) {
        *reinterpret_cast<uint4*>(o + column(0)) =
            make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (column(k) < p.n) o[column(k)] = __float2bfloat16_rn(v[k]);
      }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) red[warp][column(k) - c0] = sum[k];
  __syncthreads();
  const int c = c0 + (int)threadIdx.x;
  if (c < p.n) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kGradWarps; ++k) v += red[k][threadIdx.x];
    p.sums[(long long)blockIdx.y * p.n + c] = v;
  }
}

struct FinishParams {
  const float* part;  // [splits][M][pitch]
  int splits;
  long long M;
  int N, pitch;
  void* dw;
  long long ld_dw;
  const float* sums;  // [blocks][n]
  int blocks, n;
  float* dbias;
  int dw_ctas;        // the first CTAs add dw's parts
};

// Adds the parts of dw (four columns a thread) and, 32 columns a CTA, the blocks of dbias.
template <typename TG>
__global__ void __launch_bounds__(256) finish_kernel(const FinishParams p) {
  __shared__ float red[8][32];
  grid_dep_wait();
  if ((int)blockIdx.x < p.dw_ctas) {
    const int per_row = p.pitch / 4;
    const long long plane = p.M * p.pitch, pieces = p.M * per_row;
    const bool vec = sizeof(TG) == 4 && p.N % 4 == 0 && p.ld_dw % 4 == 0 && reinterpret_cast<uintptr_t>(p.dw) % 16 == 0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces;
         i += (long long)p.dw_ctas * 256) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int s = 0; s < p.splits; ++s) {
        const float4 t = __ldcs(reinterpret_cast<const float4*>(p.part + s * plane + i * 4));
        v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
      }
      const long long row = i / per_row;
      const int c = (int)(i - row * per_row) * 4;
      TG* to = static_cast<TG*>(p.dw) + row * p.ld_dw + c;
      if (vec) {
        *reinterpret_cast<float4*>(to) = v;
      } else {
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < p.N) put(to + k, e[k]);
      }
    }
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = ((int)blockIdx.x - p.dw_ctas) * 32 + lane;
  float v = 0.f;
  if (c < p.n)
    for (int b = warp; b < p.blocks; b += 8) v += p.sums[(long long)b * p.n + c];
  red[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && c < p.n) {
#pragma unroll
    for (int k = 1; k < 8; ++k) v += red[k][lane];
    p.dbias[c] = v;
  }
}

// ---- host side ----

constexpr int kMostRows = 0x7fffffff - 1024;

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// Rows that TMA can read as they are.
bool tma_rows(const void* p, long long ld, int size) { return bits(p) % 16 == 0 && ld * size % 16 == 0; }

// Rows that TMA can write: a store is cut off at whole 16 bytes, and what is behind a row's end is
// nobody's to write.
bool tma_out(const void* p, long long ld, int cols, int size) {
  return tma_rows(p, ld, size) && (long long)cols * size % 16 == 0;
}

long long pitch_of(int cols, int size) { return ((long long)cols * size + 15) / 16 * 16 / size; }

long long part_pitch(int cols) { return (cols + 3) / 4 * 4; }  // fp32 values between rows of parts

int64_t round_up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Map of rows [rows][cols] of elements of `size` bytes (bf16, or 8-bit), `ld` apart: boxes of
// 128 bytes by box_rows, 128-byte swizzle.
bool map_rows(CUtensorMap* map, const void* base, int size, uint64_t cols, uint64_t rows, uint64_t ld,
              uint32_t box_rows) {
  return encode_rows_map(map, base, size, cols, rows, ld * size, 128u / size, box_rows);
}

// Tiles of the result: columns of a tile and how many tiles there are.
struct Tiles {
  bool pair;
  int tile_n, m_tiles, n_tiles;
  int split = 1;  // CTAs that share a tile's reduction
};
// (whole boxes of 32 columns; on pairs tcgen05 takes 32, 64, ... 256)
int even_part(int n, int parts) { return ((n + parts - 1) / parts + 31) / 32 * 32; }

// The width and form of the tiles that leave the longest-running CTA or pair the least to do, in
// clocks, as measured: a step takes 2 clocks a column on a pair (what the tensor cores need; shared
// memory, 128 bytes of operands in and out a clock, 256 + n), 2.4 on a CTA alone, and at least
// 300 to 350; 14 a column go to storing a tile beside them; 5,700 to the beginning and end. A reduction
// that a cluster shares costs 5,000 clocks more and 55 to 105 a column for the meeting of 128 rows' sums. (us:
// 5,003 x 1,001 to 777 in 80 tiles of 256 x 208 on 76 pairs 32, in 60 of 256 x 264 23; 64 x 4,096 to 1,024
// in 32 tiles 12.6, shared by four 9.2; 33 x 1,024 to 4,096 in 128 tiles 7.9, in 43 5.7.)
Tiles pick_tiles(long long M, int N, int steps, bool may_split, int sms) {
  Tiles best{};
  double least = 1e300;
  const double met = M < 128 ? (M + 31) / 32 / 4.0 : 1.0;  // rows of a tile that there are
  for (int pair = 0; pair < 2; ++pair) {
    const long long rows = pair ? 256 : 128, m = (M + rows - 1) / rows, units = pair ? sms / 2 : sms;
    for (int n = 256; n > 0; n -= 32) {
      if (n != even_part(N, (N + n - 1) / n)) continue;  // as many tiles fit narrower ones
      const long long tiles = m * ((N + n - 1) / n), waves = (tiles + units - 1) / units;
      const double step = pair ? std::max(350.0, std::max(2.0 * n, 256.0 + n)) : std::max(300.0, 2.4 * n);
      auto take = [&](double cost, int split) {
        if (cost >= least * 0.98) return;
        least = cost;
        best.pair = pair != 0;
        best.tile_n = n;
        best.m_tiles = (int)m;
        best.n_tiles = (N + n - 1) / n;
        best.split = split;
      };
      take(waves * (std::max(step * steps, 14.0 * n) + 200.0) + 5700.0 + 4.0 * n + 25.0 * std::min(tiles, units), 1);
      // a cluster to a tile where all of them find a place at once (120 CTAs of 152 in clusters of 8, 144 in
      // those of 4)
      int log = 1;
      for (int split = 2; may_split && !pair && split <= 8 && 4 * split <= steps; split *= 2, ++log)
        if (tiles * split <= sms * (split == 8 ? 15 : split == 4 ? 18 : 19) / 19)
          take(step * ((steps + split - 1) / split) + 10700.0 + (30.0 + 25.0 * log) * n * met, split);
      if (tiles > 4 * units) break;  // narrower tiles only cost more
    }
  }
  return best;
}

// The same for dw, whose reduction can be split into parts: their sums cost a second kernel
// (4,000 clocks) and the bytes of the parts (16 a clock and SM, written and read).
Tiles pick_weight_tiles(long long M, int N, int steps, int sms, int* splits) {
  Tiles best{};
  double least = 1e300;
  *splits = 1;
  for (int pair = 0; pair < 2; ++pair) {
    const long long rows = pair ? 256 : 128, m = (M + rows - 1) / rows, units = pair ? sms / 2 : sms;
    for (int n = 256; n > 0; n -= 32) {
      if (n != even_part(N, (N + n - 1) / n)) continue;
      const int held = (n / (pair ? 2 : 1) + 63) / 64 * 64;  // columns of the blocks in shared memory
      const long long tiles = m * ((N + n - 1) / n);
      const double step = pair ? std::max(2.0 * n, 256.0 + held + n / 2) : 256.0 + held + n;
      for (int s = 1; s <= 64 && s <= (steps + 3) / 4; ++s) {
        const long long waves = (tiles * s + units - 1) / units;
        const double cost = waves * (step * ((steps + s - 1) / s) * 1.06 + 600.0 + 4.0 * n) + 1500.0 +
                            (s > 1 ? 4000.0 + 2.0 * s * (double)M * N * 4.0 / 16.0 / sms : 0.0);
        if (cost < least * 0.98) {
          least = cost;
          best.pair = pair != 0;
          best.tile_n = n;
          best.m_tiles = (int)m;
          best.n_tiles = (N + n - 1) / n;
          *splits = s;
        }
        if (tiles * s > 4 * units) break;
      }
      if (tiles > 8 * units) break;
    }
  }
  return best;
}

// The result's side of a launch: maps of its rows, the residual's and z's where TMA can take
// all of them.
struct Out {
  bool wide;
  CUtensorMap out, res, z;
};
template <typename TO>
bool map_out(Out* o, const Params& p) {
  constexpr int size = sizeof(TO), box = 64 / size;
  auto fits = [&](const void* q, long long ld, int bytes) { return !q || tma_out(q, ld, p.own_rows ? 16 : p.N, bytes); };
  o->wide = fits(p.out, p.ld_out, size) && fits(p.residual, p.ld_res, size) && fits(p.z, p.ld_z, 2);
  if (!o->wide) return true;
  const uint64_t plane = (uint64_t)(p.splits > 1 ? p.M : 1) * p.ld_out * size;
  if (!encode_box_map(&o->out, p.out, size, p.N, p.M, p.splits, p.ld_out * size, plane, box, 64)) return false;
  o->res = o->z = o->out;
  if (p.residual && !encode_box_map(&o->res, p.residual, size, p.N, p.M, 1, p.ld_res * size, p.ld_res * size, box, 64))
    return false;
  return !p.z || encode_box_map(&o->z, p.z, 2, p.N, p.M, 1, p.ld_z * 2, p.ld_z * 2, box, size == 2 ? 64 : 0);
}

template <int KIND, typename TO>
cudaError_t launch_gemm(const CUtensorMap& a, const CUtensorMap& b, Params p, const Tiles& t, int sms,
                        cudaStream_t s) {
  Out o{};
  if (KIND != kWeight) p.splits = 1;
  if (!map_out<TO>(&o, p)) return cudaErrorInvalidValue;
  const bool wide = o.wide;
  const bool split = KIND != kWeight && wide && t.split > 1;
  const int ctas = t.pair ? 2 : split ? t.split : 1;
  const int n = t.tile_n / (t.pair ? 2 : 1);
  p.tile_n = t.tile_n;
  p.m_tiles = t.m_tiles;
  p.n_tiles = t.n_tiles;
  p.stage_bytes = 16384u + (KIND >= kInput ? (uint32_t)((n + 63) / 64) * 8192u : ((uint32_t)n * 128u + 1023u) / 1024u * 1024u);
  p.two = !split && (p.residual || p.steps <= 8 || (p.gelu && p.steps < 32));
  p.boxes = (p.two ? 2u : 1u) + (p.z ? 1u : 0u);
  const uint32_t beside =
      1024u + (kBars + 1) * 8u + 16u + kColumns + (wide ? kEpiWarps * p.boxes * kBox : kStagingOdd);
  p.stages = (int)std::min<uint32_t>(kMaxStages, (kSmemMax - beside) / p.stage_bytes);
  const uint32_t smem = beside + (uint32_t)p.stages * p.stage_bytes;
  p.sum_steps = KIND == kWeight || (KIND != kInput && sizeof(TO) == 4) ? kSumSteps : kSumSteps16;
  p.wait_limit = gemm_wait_limit();
  void (*kernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                 const Params) =
      t.pair ? (wide ? gemm_kernel<KIND, TO, true, true, false> : gemm_kernel<KIND, TO, true, false, false>)
             : (wide ? gemm_kernel<KIND, TO, false, true, false> : gemm_kernel<KIND, TO, false, false, false>);
  if constexpr (KIND != kWeight) {
    if (split) {
      kernel = gemm_kernel<KIND, TO, false, true, true>;
      p.splits = t.split;
    }
  } else if (p.live) {
    kernel = t.pair ? (wide ? gemm_kernel<KIND, TO, true, true, true> : gemm_kernel<KIND, TO, true, false, true>)
                    : (wide ? gemm_kernel<KIND, TO, false, true, true> : gemm_kernel<KIND, TO, false, false, true>);
  }
  const cudaError_t e = allow_smem_once(kernel, smem);
  if (e != cudaSuccess) return e;
  const long long items = (long long)t.m_tiles * t.n_tiles * (split ? 1 : p.splits);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas * (split ? items : std::min<long long>(items, sms / ctas))));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, b, o.out, o.res, o.z, p);
}

template <int SIZE, int NT, typename TO>
cudaError_t launch_rows_as(const RowsParams& p, bool vec, cudaStream_t s) {
  const int blocks = (p.bytes + 127) / 128;
  const int warps = std::min(kRowsWarps, std::max(4, (blocks + 1) / 2));
  void (*kernel)(const RowsParams) = vec ? rows_kernel<SIZE, NT, true, TO> : rows_kernel<SIZE, NT, false, TO>;
  return launch_dependent(kernel, dim3((p.e.N + 15) / 16), dim3(32 * warps), 0, s, p);
}
template <int SIZE, typename TO>
cudaError_t launch_rows(const RowsParams& p, bool vec, cudaStream_t s) {
  if (p.e.M <= 8) return launch_rows_as<SIZE, 1, TO>(p, vec, s);
  if (p.e.M <= 16) return launch_rows_as<SIZE, 2, TO>(p, vec, s);
  return launch_rows_as<SIZE, 4, TO>(p, vec, s);
}

cudaError_t launch_layout(const Rows& a, const Rows& b, int size, int sms, cudaStream_t s) {
  const long long warps = a.warps() + b.warps();
  if (warps == 0) return cudaSuccess;
  const int grid = (int)std::min<long long>((warps + 7) / 8, 8ll * sms);
  return launch_dependent(size == 2 ? layout_kernel<uint16_t> : layout_kernel<uint8_t>, dim3(grid), dim3(256), 0, s,
                          a, b);
}

int check(const unif_moe_linear* p) {
  if (!p) { set_error("the description is NULL"); return UNIF_MOE_ERR_ARG; }
  if (p->rows < 0 || p->rows > kMostRows || p->cols < 1 || p->n < 1 || p->cols > UNIF_MOE_LINEAR_MAX_COLS ||
      p->n > UNIF_MOE_LINEAR_MAX_COLS) {
    set_error("bad sizes: rows=%lld cols=%d n=%d", (long long)p->rows, p->cols, p->n);
    return UNIF_MOE_ERR_ARG;
  }
  auto type = [](int t) { return t == UNIF_MOE_F32 || t == UNIF_MOE_BF16; };
  if ((p->in_dtype != UNIF_MOE_BF16 && p->in_dtype != UNIF_MOE_E4M3) || !type(p->out_dtype) ||
      !type(p->bias_dtype) || p->activation < UNIF_MOE_ACTIVATION_NONE ||
      p->activation > UNIF_MOE_ACTIVATION_GELU) {
    set_error("bad dtypes (in %d, out %d, bias %d) or activation %d", p->in_dtype, p->out_dtype, p->bias_dtype,
              p->activation);
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

bool few_rows(const unif_moe_linear* p) {
  return p->rows <= kRowsMax && (int64_t)p->cols * (p->in_dtype == UNIF_MOE_BF16 ? 2 : 1) <= kRowsBytes;
}

int in_size(const unif_moe_linear* p) { return p->in_dtype == UNIF_MOE_BF16 ? 2 : 1; }

int64_t forward_bytes(const unif_moe_linear* p, const void* x, long long ld_x, const void* w, long long ld_w) {
  const int size = in_size(p);
  if (few_rows(p)) return 0;
  int64_t need = 0;
  if (!tma_rows(x, ld_x, size)) need += round_up(p->rows * pitch_of(p->cols, size) * size);
  if (!tma_rows(w, ld_w, size)) need += round_up((int64_t)p->n * pitch_of(p->cols, size) * size);
  return need;
}

// The workspace of a backward: where each part begins.
struct Plan {
  int sms, splits, blocks, per;
  bool copy_x, copy_w, make_dz, sums, list;
  long long px, pw, pz;  // pitches
  int64_t x, w, dz, part, bias, live, dead, total;
  Tiles in, weight;
};
Plan plan_backward(const unif_moe_linear* p, const unif_moe_linear_grad* g, int sms) {
  Plan r{};
  r.sms = sms;
  const long long T = p->rows;
  r.copy_x = g->dw_dev && !tma_rows(g->x_dev, g->ld_x, 2);
  r.copy_w = g->dx_dev && !tma_rows(g->w_dev, g->ld_w, 2);
  r.make_dz = (g->dx_dev || g->dw_dev) &&
              (p->activation != UNIF_MOE_ACTIVATION_NONE || g->dout_dtype != UNIF_MOE_BF16 ||
               !tma_rows(g->dout_dev, g->ld_dout, 2));
  r.sums = g->dbias_dev != nullptr;
  r.px = r.copy_x ? pitch_of(p->cols, 2) : g->ld_x;
  r.pw = r.copy_w ? pitch_of(p->cols, 2) : g->ld_w;
  r.pz = r.make_dz ? pitch_of(p->n, 2) : g->ld_dout;
  // row blocks of grad_kernel: the three CTAs that an SM holds at once
  const long long cols = (p->n + 255) / 256, most = std::max<long long>(1, 3ll * sms / cols);
  r.per = (int)std::max<long long>(kGradWarps * kGradRows, (T + most - 1) / most);
  r.blocks = (int)((T + r.per - 1) / r.per);
  r.in = pick_tiles(T, p->cols, (p->n + 63) / 64, tma_out(g->dx_dev, g->ld_dx, p->cols, 2), sms);
  const int steps = (int)((T + 63) / 64);
  r.weight = pick_weight_tiles(p->n, p->cols, steps, sms, &r.splits);
  int64_t at = 0;
  auto take = [&](bool want, int64_t bytes) {
    const int64_t here = at;
    if (want) at += round_up(bytes);
    return here;
  };
  r.x = take(r.copy_x, T * r.px * 2);
  r.w = take(r.copy_w, (int64_t)p->n * r.pw * 2);
  r.dz = take(r.make_dz, T * r.pz * 2);
  r.part = take(g->dw_dev && r.splits > 1, (int64_t)r.splits * p->n * part_pitch(p->cols) * 4);
  r.bias = take(r.sums, (int64_t)r.blocks * p->n * 4);
  r.list = g->dw_dev && g->token_mask_dev;
  r.live = take(r.list, 4 * (int64_t)(steps + 1));
  r.dead = take(r.list, 8 * (int64_t)steps);
  r.total = at;
  return r;
}

int check_grad(const unif_moe_linear* p, const unif_moe_linear_grad* g) {
  const int rc = check(p);
  if (rc != UNIF_MOE_OK) return rc;
  if (!g) { set_error("the gradients' description is NULL"); return UNIF_MOE_ERR_ARG; }
  auto type = [](int t) { return t == UNIF_MOE_F32 || t == UNIF_MOE_BF16; };
  if (p->in_dtype != UNIF_MOE_BF16 || !type(g->dout_dtype) || !type(g->grad_dtype)) {
    set_error("gradients are those of bf16 rows; bad dtypes (in %d, dout %d, gradient %d)", p->in_dtype,
              g->dout_dtype, g->grad_dtype);
    return UNIF_MOE_ERR_ARG;
  }
  const bool act = p->activation != UNIF_MOE_ACTIVATION_NONE;
  if (p->rows > 0 && ((!g->x_dev && g->dw_dev) || (!g->w_dev && g->dx_dev) || !g->dout_dev || (act && !g->z_dev))) {
    set_error("x, w, dout or z is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if ((g->dw_dev && (g->ld_dw < p->cols || (p->rows > 0 && g->ld_x < p->cols))) ||
      (p->rows > 0 && ((g->dx_dev && (g->ld_w < p->cols || g->ld_dx < p->cols)) || g->ld_dout < p->n ||
                       (act && g->ld_z < p->n)))) {
    set_error("a row stride is below the width");
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

}  // namespace lin
}  // namespace unif

using unif::set_error;
namespace ln = unif::lin;

#define UNIF_LAUNCH(call)                                             \
  do {                                                                \
    const cudaError_t e_ = (call);                                    \
    if (e_ != cudaSuccess) {                                          \
      set_error("linear: %s", cudaGetErrorString(e_));                \
      return UNIF_MOE_ERR_CUDA;                                       \
    }                                                                 \
  } while (0)

extern "C" {

int64_t unif_moe_linear_workspace(const unif_moe_linear* p, const void* x, int64_t ld_x, const void* w,
                                  int64_t ld_w) {
  set_error("%s", "");
  if (ln::check(p) != UNIF_MOE_OK) return -1;
  return ln::forward_bytes(p, x, ld_x, w, ld_w);
}

int unif_moe_linear_forward(const unif_moe_linear* p, const void* x, int64_t ld_x, const float* x_scale,
                            const void* w, int64_t ld_w, const float* w_scale, const void* bias,
                            const void* residual, int64_t ld_res, const uint8_t* mask, void* out, int64_t ld_out,
                            void* z, int64_t ld_z, void* workspace, int64_t workspace_bytes, int32_t* status,
                            void* stream) {
  set_error("%s", "");
  const int rc = ln::check(p);
  if (rc != UNIF_MOE_OK || p->rows == 0) return rc;
  if (!x || !w || !out || !status) {
    set_error("x, w, out or status is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (p->in_dtype == UNIF_MOE_BF16 && (x_scale || w_scale)) {
    set_error("bf16 rows take no scales");
    return UNIF_MOE_ERR_ARG;
  }
  if (ld_x < p->cols || ld_w < p->cols || ld_out < p->n || (residual && ld_res < p->n) || (z && ld_z < p->n)) {
    set_error("a row stride is below the width");
    return UNIF_MOE_ERR_ARG;
  }
  const int size = ln::in_size(p), os = p->out_dtype == UNIF_MOE_F32 ? 4 : 2;
  const int64_t need = ln::forward_bytes(p, x, ld_x, w, ld_w);
  if (need > workspace_bytes || (need && !workspace)) {
    set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (need && ln::bits(workspace) % 16) {
    set_error("the workspace must be 16-byte aligned");
    return UNIF_MOE_ERR_ARG;
  }
  auto rows_of = [&](const void* q, int64_t ld, int64_t cols, int64_t rows, int bytes) {
    return unif::Block{q, ld * bytes, cols * bytes, rows};
  };
  const unif::Block to = rows_of(out, ld_out, p->n, p->rows, os), res = rows_of(residual, ld_res, p->n, p->rows, os),
                    kept = rows_of(z, ld_z, p->n, p->rows, 2), bx = rows_of(x, ld_x, p->cols, p->rows, size),
                    bw = rows_of(w, ld_w, p->cols, p->n, size),
                    bb = unif::flat(bias, p->n * (p->bias_dtype == UNIF_MOE_F32 ? 4ll : 2ll)),
                    bsx = unif::flat(x_scale, p->rows * 4), bsw = unif::flat(w_scale, p->n * 4ll),
                    bm = unif::flat(mask, p->rows), ws_used = unif::flat(workspace, need), st = unif::flat(status, 4);
  const bool in_place = out == residual && (ld_out == ld_res || p->rows == 1);
  if (unif::overlap_any(to, {bx, bw, kept, bb, bsx, bsw, bm, ws_used, st}) || (!in_place && unif::overlap(to, res)) ||
      unif::overlap_any(kept, {bx, bw, res, bb, bsx, bsw, bm, ws_used, st})) {
    set_error("out or z overlaps another array of the call (the residual in out's place excepted)");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  ln::Params e{};
  e.M = (int)p->rows;
  e.N = p->n;
  e.splits = 1;
  e.gelu = p->activation == UNIF_MOE_ACTIVATION_GELU;
  e.out = out;
  e.ld_out = ld_out;
  e.sm = x_scale;
  e.sn = w_scale;
  e.bias = bias;
  e.bias_f32 = p->bias_dtype == UNIF_MOE_F32;
  e.residual = residual;
  e.ld_res = ld_res;
  e.mask = mask;
  e.z = static_cast<__nv_bfloat16*>(z);
  e.ld_z = ld_z;
  e.status = status;
  if (ln::few_rows(p)) {
    ln::RowsParams r{};
    r.e = e;
    r.x = static_cast<const uint8_t*>(x);
    r.w = static_cast<const uint8_t*>(w);
    r.ld_x = ld_x * size;
    r.ld_w = ld_w * size;
    r.bytes = p->cols * size;
    const bool vec = ln::tma_rows(x, ld_x, size) && ln::tma_rows(w, ld_w, size);
    if (size == 2)
      UNIF_LAUNCH(os == 4 ? (ln::launch_rows<2, float>(r, vec, s)) : (ln::launch_rows<2, __nv_bfloat16>(r, vec, s)));
    else
      UNIF_LAUNCH(os == 4 ? (ln::launch_rows<1, float>(r, vec, s)) : (ln::launch_rows<1, __nv_bfloat16>(r, vec, s)));
    return UNIF_MOE_OK;
  }
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  long long px = ld_x, pw = ld_w;
  ln::Rows copies[2] = {};
  if (!ln::tma_rows(x, ld_x, size)) {
    px = ln::pitch_of(p->cols, size);
    copies[0] = {x, ld_x, ws, px, p->rows, p->cols, nullptr};
    x = ws;
    ws += ln::round_up(p->rows * px * size);
  }
  if (!ln::tma_rows(w, ld_w, size)) {
    pw = ln::pitch_of(p->cols, size);
    copies[1] = {w, ld_w, ws, pw, p->n, p->cols, nullptr};
    w = ws;
  }
  UNIF_LAUNCH(ln::launch_layout(copies[0], copies[1], size, sms, s));
  const int steps = (int)(((int64_t)p->cols * size + 127) / 128);
  const bool wide = ln::tma_out(out, ld_out, p->n, os) && (!residual || ln::tma_out(residual, ld_res, p->n, os)) &&
                    (!z || ln::tma_out(z, ld_z, p->n, 2));
  const ln::Tiles t = ln::pick_tiles(p->rows, p->n, steps, wide, sms);
  if ((long long)t.m_tiles * t.n_tiles > 0x7fff0000) {
    set_error("too many tiles: rows=%lld n=%d", (long long)p->rows, p->n);
    return UNIF_MOE_ERR_SHAPE;
  }
  e.steps = steps;
  CUtensorMap a, b;
  if (!ln::map_rows(&a, x, size, p->cols, p->rows, px, 128) ||
      !ln::map_rows(&b, w, size, p->cols, p->n, pw, t.tile_n / (t.pair ? 2 : 1))) {
    set_error("cuTensorMapEncodeTiled failed");
    return UNIF_MOE_ERR_CUDA;
  }
  if (size == 2)
    UNIF_LAUNCH(os == 4 ? (ln::launch_gemm<ln::kForward, float>(a, b, e, t, sms, s))
                        : (ln::launch_gemm<ln::kForward, __nv_bfloat16>(a, b, e, t, sms, s)));
  else
    UNIF_LAUNCH(os == 4 ? (ln::launch_gemm<ln::kForward8, float>(a, b, e, t, sms, s))
                        : (ln::launch_gemm<ln::kForward8, __nv_bfloat16>(a, b, e, t, sms, s)));
  return UNIF_MOE_OK;
}

int64_t unif_moe_linear_backward_workspace(const unif_moe_linear* p, const unif_moe_linear_grad* g) {
  set_error("%s", "");
  int sms = 0;
  if (ln::check_grad(p, g) != UNIF_MOE_OK || unif::sm_count(&sms) != UNIF_MOE_OK) return -1;
  return p->rows == 0 ? 0 : ln::plan_backward(p, g, sms).total;
}

int unif_moe_linear_backward(const unif_moe_linear* p, const unif_moe_linear_grad* g, void* workspace,
                             int64_t workspace_bytes, int32_t* status, void* stream) {
  set_error("%s", "");
  const int rc = ln::check_grad(p, g);
  if (rc != UNIF_MOE_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int gs = g->grad_dtype == UNIF_MOE_F32 ? 4 : 2;
  if (p->rows == 0) {
    if (g->dw_dev)
      UNIF_LAUNCH(cudaMemset2DAsync(g->dw_dev, (size_t)g->ld_dw * gs, 0, (size_t)p->cols * gs, p->n, s));
    if (g->dbias_dev) UNIF_LAUNCH(cudaMemsetAsync(g->dbias_dev, 0, sizeof(float) * p->n, s));
    return UNIF_MOE_OK;
  }
  if (!status) { set_error("status is NULL"); return UNIF_MOE_ERR_ARG; }
  if (!g->dx_dev && !g->dw_dev && !g->dbias_dev) return UNIF_MOE_OK;
  // what is not read (x without dw, w without dx, z without an activation) may lie anywhere
  auto rows_of = [](const void* q, int64_t ld, int64_t cols, int64_t rows, int64_t bytes) {
    return unif::Block{q, ld * bytes, cols * bytes, rows};
  };
  const unif::Block bx = rows_of(g->dw_dev ? g->x_dev : nullptr, g->ld_x, p->cols, p->rows, 2),
                    bw = rows_of(g->dx_dev ? g->w_dev : nullptr, g->ld_w, p->cols, p->n, 2),
                    bd = rows_of(g->dout_dev, g->ld_dout, p->n, p->rows, g->dout_dtype == UNIF_MOE_F32 ? 4 : 2),
                    bz = rows_of(p->activation != UNIF_MOE_ACTIVATION_NONE ? g->z_dev : nullptr, g->ld_z, p->n, p->rows, 2),
                    bm = unif::flat(g->token_mask_dev, p->rows), st = unif::flat(status, 4),
                    dx = rows_of(g->dx_dev, g->ld_dx, p->cols, p->rows, 2),
                    dw = rows_of(g->dw_dev, g->ld_dw, p->cols, p->n, gs), db = unif::flat(g->dbias_dev, p->n * 4ll);
  if (unif::overlap_any(dx, {bx, bw, bd, bz, bm, st, dw, db}) ||
      unif::overlap_any(dw, {bx, bw, bd, bz, bm, st, db}) ||
      unif::overlap_any(db, {bx, bw, bd, bz, bm, st})) {
    set_error("dx, dw or dbias overlaps another array of the call");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rs = unif::sm_count(&sms);
  if (rs != UNIF_MOE_OK) return rs;
  const ln::Plan pl = ln::plan_backward(p, g, sms);
  if (pl.total > workspace_bytes || (pl.total && !workspace)) {
    set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)pl.total);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (pl.total && ln::bits(workspace) % 32) {
    set_error("the workspace must be 32-byte aligned");
    return UNIF_MOE_ERR_ARG;
  }
  if (unif::overlap_any(unif::flat(workspace, pl.total), {dx, dw, db})) {
    set_error("dx, dw or dbias overlaps the workspace");
    return UNIF_MOE_ERR_ARG;
  }
  if ((long long)pl.in.m_tiles * pl.in.n_tiles > 0x7fff0000 ||
      (long long)pl.weight.m_tiles * pl.weight.n_tiles * pl.splits > 0x7fff0000) {
    set_error("too many tiles: rows=%lld cols=%d n=%d", (long long)p->rows, p->cols, p->n);
    return UNIF_MOE_ERR_SHAPE;
  }
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const void *x = g->x_dev, *w = g->w_dev, *dz = g->dout_dev;
  ln::Rows copies[2] = {};
  if (pl.copy_x) {
    x = ws + pl.x;
    copies[0] = {g->x_dev, g->ld_x, ws + pl.x, pl.px, p->rows, p->cols, g->token_mask_dev};
  }
  if (pl.copy_w) {
    w = ws + pl.w;
    copies[1] = {g->w_dev, g->ld_w, ws + pl.w, pl.pw, p->n, p->cols, nullptr};
  }
  UNIF_LAUNCH(ln::launch_layout(copies[0], copies[1], 2, sms, s));
  if (pl.list)
    UNIF_LAUNCH(unif::launch_dependent(ln::steps_kernel, dim3(1), dim3(ln::kListThreads), 0, s, g->token_mask_dev,
                                       (long long)p->rows, pl.splits, reinterpret_cast<int*>(ws + pl.live),
                                       reinterpret_cast<unsigned long long*>(ws + pl.dead)));
  if (pl.make_dz || pl.sums) {
    ln::GradParams q{};
    q.rows = p->rows;
    q.n = p->n;
    q.per = pl.per;
    q.dout = g->dout_dev;
    q.ld_dout = g->ld_dout;
    q.z = p->activation != UNIF_MOE_ACTIVATION_NONE ? static_cast<const __nv_bfloat16*>(g->z_dev) : nullptr;
    q.ld_z = g->ld_z;
    q.mask = g->token_mask_dev;
    if (pl.make_dz) {
      dz = ws + pl.dz;
      q.dz = reinterpret_cast<__nv_bfloat16*>(ws + pl.dz);
      q.ld_dz = pl.pz;
    }
    q.sums = pl.sums ? reinterpret_cast<float*>(ws + pl.bias) : nullptr;
    const int ds = g->dout_dtype == UNIF_MOE_F32 ? 4 : 2;
    const bool vec = p->n % 8 == 0 && ln::bits(g->dout_dev) % 16 == 0 && g->ld_dout * ds % 16 == 0 &&
                     (!q.z || ln::tma_rows(g->z_dev, g->ld_z, 2));
    const dim3 grid((p->n + 255) / 256, pl.blocks), block(32 * ln::kGradWarps);
    void (*kernel)(const ln::GradParams) =
        ds == 4 ? (vec ? ln::grad_kernel<float, true> : ln::grad_kernel<float, false>)
                : (vec ? ln::grad_kernel<__nv_bfloat16, true> : ln::grad_kernel<__nv_bfloat16, false>);
    UNIF_LAUNCH(unif::launch_dependent(kernel, grid, block, 0, s, q));
  }
  if (g->dx_dev) {
    ln::Params e{};
    e.M = (int)p->rows;
    e.N = p->cols;
    e.splits = 1;
    e.steps = (p->n + 63) / 64;
    e.mask = g->token_mask_dev;  // (dz's padding rows are 0, but 0 times an infinite weight is not)
    e.out = g->dx_dev;
    e.ld_out = g->ld_dx;
    e.status = status;
    CUtensorMap a, b;
    if (!ln::map_rows(&a, dz, 2, p->n, p->rows, pl.pz, 128) || !ln::map_rows(&b, w, 2, p->cols, p->n, pl.pw, 64)) {
      set_error("cuTensorMapEncodeTiled failed");
      return UNIF_MOE_ERR_CUDA;
    }
    UNIF_LAUNCH((ln::launch_gemm<ln::kInput, __nv_bfloat16>(a, b, e, pl.in, sms, s)));
  }
  if (g->dw_dev) {
    ln::Params e{};
    e.M = p->n;
    e.N = p->cols;
    e.splits = pl.splits;
    e.steps = (int)((p->rows + 63) / 64);
    // parts of the sum go to the workspace
    e.out = pl.splits > 1 ? ws + pl.part : g->dw_dev;
    e.ld_out = pl.splits > 1 ? ln::part_pitch(p->cols) : g->ld_dw;
    e.own_rows = pl.splits > 1;
    e.clean_a = !pl.make_dz;
    e.clean_b = !pl.copy_x;
    if (pl.list) {
      e.live = reinterpret_cast<const int*>(ws + pl.live);
      e.dead = reinterpret_cast<const unsigned long long*>(ws + pl.dead);
    }
    e.status = status;
    CUtensorMap a, b;
    if (!ln::map_rows(&a, dz, 2, p->n, p->rows, pl.pz, 64) || !ln::map_rows(&b, x, 2, p->cols, p->rows, pl.px, 64)) {
      set_error("cuTensorMapEncodeTiled failed");
      return UNIF_MOE_ERR_CUDA;
    }
    UNIF_LAUNCH(gs == 4 || pl.splits > 1 ? (ln::launch_gemm<ln::kWeight, float>(a, b, e, pl.weight, sms, s))
                                         : (ln::launch_gemm<ln::kWeight, __nv_bfloat16>(a, b, e, pl.weight, sms, s)));
  }
  const bool add = g->dw_dev && pl.splits > 1;
  if (add || pl.sums) {
    ln::FinishParams q{};
    q.part = reinterpret_cast<const float*>(ws + pl.part);
    q.splits = pl.splits;
    q.M = p->n;
    q.N = p->cols;
    q.pitch = (int)ln::part_pitch(p->cols);
    q.dw = g->dw_dev;
    q.ld_dw = g->ld_dw;
    q.sums = reinterpret_cast<const float*>(ws + pl.bias);
    q.blocks = pl.blocks;
    q.n = p->n;
    q.dbias = g->dbias_dev;
    q.dw_ctas = add ? (int)std::min<int64_t>(((int64_t)p->n * p->cols + 1023) / 1024, 8ll * sms) : 0;
    const unsigned grid = q.dw_ctas + (pl.sums ? (p->n + 31) / 32 : 0);
    void (*kernel)(const ln::FinishParams) = gs == 4 ? ln::finish_kernel<float> : ln::finish_kernel<__nv_bfloat16>;
    UNIF_LAUNCH(unif::launch_dependent(kernel, dim3(grid), dim3(256), 0, s, q));
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

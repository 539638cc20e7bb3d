// Product of rows in MXFP4 with the weights of their group, also in MXFP4
// (unif_moe_mxfp4_product): out[r][n] = act(sum_c A[r][c] W[g(r)][n][c]).
//
// What bounds it: with few rows the weights' bytes (24 rows in 33 groups of 4,096 x 1,024:
// 11.3 us, 4.8 TB/s); with many steps shared memory for the larger part: it takes 28 KB of a
// step's operands in and gives 28 KB to the MMAs, 448 clocks at 128 bytes a clock, of about 710
// that a step takes (131,072 rows of 1,024 x 4,096 in 33 groups, fp32 output, 245 us back to back
// at 1,720 MHz under the power cap: 37 items of 16 steps a pair; 230 us, 4.8 PFLOP/s, with
// pauses; the bytes need 131); no counter shows the rest; with few steps the stores and GELU of a tile beside
// the next tile's loads (100,003 rows of 192 x 768 in 272 groups: 23.3 us, 4.2 TB/s).
//
// tcgen05 block-scaled MMAs (kind mxf4: products of 4-bit elements and 8-bit
// scales exact, sums in fp32 in TMEM). The weights are the M operand, 128 output
// channels to a tile, and the rows the N operand, up to 192 to a tile: a tile
// of few rows then costs few columns, whatever a group's size, and a lane of
// the accumulator is a channel, so that 32 lanes store consecutive channels of
// one row. (Where groups are large, rows can be M: see the rule at the launch.)
//
// One CTA per SM, or a pair of CTAs per two SMs, walks (row tile, channel tile) items, steps of 256 columns
// through a ring of stages. Roles of the warps: 8 store accumulators, one loads
// codes by TMA, one issues MMAs, 4 bring the scales: eight bytes a row and step,
// read from row-major storage into registers and written as the 512-byte blocks
// that tcgen05.cp spreads over TMEM (byte 16 (r % 32) + 4 (r / 32) + b of a block
// is scale b of row r).
#include <math.h>

#include "tc_common.cuh"

namespace unif {
namespace fp4p {

using namespace tc;

constexpr int kTN = 192;         // rows of a tile (MMA N)
constexpr int kStep = 256;       // columns of a step: 128 bytes of codes, 8 scales
// Stages of the ring; fewer where the table of groups (from 324 on) needs the room.
constexpr int kMaxStages = 5, kFewStages = 3;
constexpr uint32_t kBytesW = 128 * 128;
// Row codes of a stage: the tile's rows, or with PAIR this CTA's half of them.
__host__ __device__ constexpr int stage_rows(bool pair) { return pair ? kTN / 2 : kTN; }
__host__ __device__ constexpr uint32_t stage_bytes(bool pair) {
  return kBytesW + (uint32_t)stage_rows(pair) * 128u;
}
// Scales of two steps: 512-byte blocks [step][128 columns][weights | rows 0-127, rows 128-191].
constexpr int kScaleBufs = 3;
constexpr uint32_t kBytesSW = 4 * 512, kBytesSA = 8 * 512, kBytesS = kBytesSW + kBytesSA;
constexpr int kEpiWarps = 8, kTmaWarp = 8, kMmaWarp = 9, kScaleWarp = 10, kScaleWarps = 4;
constexpr int kThreads = 32 * (kScaleWarp + kScaleWarps);
// Rows of the smaller TMA boxes of A (half of these with PAIR): one box where the
// tile has at most 16 or 64 rows or more than 128, else two of 64. (Six boxes of 32
// took the loader 970 cycles a step.)
constexpr int kBoxS = 16, kBoxM = 64;
// TMEM columns: two accumulators, then the scales of each stage.
constexpr uint32_t kAcc = kTN, kScaleCol = 2 * kTN, kScaleCols = 24, kTmemCols = 512;
static_assert(kScaleCol + kMaxStages * kScaleCols <= kTmemCols, "TMEM");
// Items of a CTA that are looked up once, by all threads together: one thread's
// search takes some 1,800 cycles, as long as an item of three steps.
constexpr int kListed = 256;
constexpr int kBars = 2 * kMaxStages + 5 + 2 * kScaleBufs;

struct Params {
  int rows, N, G, num_kb;
  const int32_t* offsets;   // [G + 1], or NULL: one group of all rows
  const uint8_t* m_scales;  // of the M operand, of the N operand
  const uint8_t* n_scales;
  int pitch;                // scale bytes of a row
  void* out;
  long long ld;
  bool pairs;               // out and ld allow stores of two bf16
  int* status;
  long long wait_limit;
};

__host__ __device__ constexpr uint32_t smem_bytes(bool pair, int stages, int G) {
  return 1024u + stages * stage_bytes(pair) + kScaleBufs * kBytesS + (kBars + 1) * 8u + kListed * 16u +
         (uint32_t)(3 * G + 1) * 4u + 32u;
}

template <bool PAIR>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                         uint32_t sa, uint32_t sb, uint32_t accumulate) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::
            "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::
            "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// A 512-byte block of scales (32 x 16 bytes) to four TMEM columns, in all four
// lane quarters; with PAIR in both CTAs, each from its own shared memory.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if (PAIR)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Descriptor of such a block: no swizzle, 8-row groups of 16-byte rows 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) |
         ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
// Instruction descriptor of kind mxf4: A and B E2M1 (bits 7-9, 10-12 = 1), N >> 3
// at bits 17-22, scales E8M0 (bit 23), M >> 7 (1, or 2 with PAIR) at bits 27-28; bits 4-5 and 29-30
// pick the byte of a TMEM word at which B's and A's scales start (0 or 2).
__device__ __forceinline__ uint32_t idesc_mxf4(bool pair, int n, int scale_byte) {
  return ((uint32_t)scale_byte << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) |
         (1u << 23) | ((pair ? 2u : 1u) << 27) | ((uint32_t)scale_byte << 29);
}

constexpr uint32_t kSmemMax = 232448;  // shared memory that a CTA can have, all of it dynamic
static_assert(smem_bytes(false, kFewStages, UNIF_MOE_MXFP4_MAX_GROUPS) <= kSmemMax, "shared memory");

__device__ __forceinline__ void wait_settle(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > limit) return;
}

// Items of the walk: up to 128 entries of the M operand (for each CTA of a pair) and
// up to kTN of the N operand; entries are rows or, of the weights, channels.
struct __align__(16) Item {
  int m0, n0;      // first entry of each operand, in its tensor; m0: this CTA's
  int ch0;         // first output channel of the tile (this CTA's, where channels are M)
  uint32_t sizes;  // entries: of M for this CTA (0 to 128), of N (1 to kTN) in the upper half
  __device__ __forceinline__ int m() const { return (int)(sizes & 0xffffu); }
  __device__ __forceinline__ int n() const { return (int)(sizes >> 16); }
};

__device__ __forceinline__ float gelu_erf(float y) {
  return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
}

// GELU(v) = v Phi(v) of two values, rounded to bf16 once. With x = -|v|, Phi(x) = 2^Q(x), Q
// of degree 11 (its fit in tests/gelu_log_fit.py), and GELU(v) = max(v, 0) + x Phi(x):
// within 2^-18 of the value for v >= -4, 2^-12 down to v = -12.9, and 0 below (where the
// value is under 2e-37), so that the rounding (2^-8 at most) decides. The layer's
// epilogue, a hardware tanh, has an error of 3e-4 |v|, which for v < -1.4 is more than the
// rounding, and at -4 more than the value. Its 12 multiply-adds a value bound the storing
// warps (100,000 rows in 33 groups of 768 x 768 44.1 us without GELU, 64.5 so, 54.2 with that
// tanh; with x^2 apart from a Q of degree 12, 15 of them, 69.6; rows as M, 100,003 rows in 272
// groups of 192 x 768 22.2, 23.3, 22.2 and 24.2). x = -13 stands for all that is smaller; NaN
// stays NaN.
#define UNIF_K2(bits) ((uint64_t)(bits##u) << 32 | (uint64_t)(bits##u))
__device__ __forceinline__ uint32_t gelu2(float v0, float v1) {
  float x0, x1, e0, e1, y0, y1;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x0) : "f"(-fabsf(v0)), "f"(-13.f));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x1) : "f"(-fabsf(v1)), "f"(-13.f));
  const uint64_t x = pk2(x0, x1);
  uint64_t q = UNIF_K2(0xae8f0e53);     // q11
  q = fma2(q, x, UNIF_K2(0xb191c94c));  // q10
  q = fma2(q, x, UNIF_K2(0xb3f84d3a));  // q9
  q = fma2(q, x, UNIF_K2(0xb5def6f2));  // q8
  q = fma2(q, x, UNIF_K2(0xb74c0539));  // q7
  q = fma2(q, x, UNIF_K2(0xb738e2e6));  // q6
  q = fma2(q, x, UNIF_K2(0x3a367766));  // q5
  q = fma2(q, x, UNIF_K2(0x3c03d9e8));  // q4
  q = fma2(q, x, UNIF_K2(0x3d5ae7de));  // q3
  q = fma2(q, x, UNIF_K2(0xbeeae20c));  // q2
  q = fma2(q, x, UNIF_K2(0x3f935a21));  // q1
  q = fma2(q, x, UNIF_K2(0xbf7fffd6));  // q0
  upk2(q, e0, e1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(e0));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(e1));
  upk2(fma2(x, pk2(e0, e1), pk2(fmaxf(v0, 0.f), fmaxf(v1, 0.f))), y0, y1);
  const __nv_bfloat162 h = __floats2bfloat162_rn(y0, y1);
  return *reinterpret_cast<const uint32_t*>(&h);
}
#undef UNIF_K2

// A row's `count` (at most 32) channels from `ch` on, one row per lane: whole
// sectors, eight 32-bit words a store. (Sixteen channels that are not all there, at the
// end of a row of odd width, are stored one by one.)
template <bool GELU>
__device__ __forceinline__ void store_row(const Params& p, float (&v)[32], int row, int ch, int count) {
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.out) + (long long)row * p.ld + ch;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = v[16 * g + 2 * j], b = v[16 * g + 2 * j + 1];
      if (GELU) {
        h[j] = gelu2(a, b);
      } else {
        __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
        h[j] = *reinterpret_cast<uint32_t*>(&t);
      }
    }
    if (16 * g + 16 <= count) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(o + 16 * g),
                   "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]), "r"(h[4]), "r"(h[5]), "r"(h[6]),
                   "r"(h[7])
                   : "memory");
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const __nv_bfloat162 t = *reinterpret_cast<__nv_bfloat162*>(&h[j]);
        if (16 * g + 2 * j < count) o[16 * g + 2 * j] = t.x;
        if (16 * g + 2 * j + 1 < count) o[16 * g + 2 * j + 1] = t.y;
      }
    }
  }
}

// The first `rows` (at most 32) rows of a chunk, one channel per lane.
template <typename TO, bool GELU>
__device__ __forceinline__ void store_chunk(const Params& p, float (&v)[32], int row0, int rows, int ch,
                                            int lane) {
  if constexpr (sizeof(TO) == 4) {
    float* o = static_cast<float*>(p.out) + (long long)row0 * p.ld + ch;
    if (ch < p.N)
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (j < rows) {
          *o = GELU ? gelu_erf(v[j]) : v[j];
        }
        o += p.ld;
      }
  } else {
    uint32_t h[16];  // rows 2 i and 2 i + 1 of this lane's channel
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (GELU) {
        h[i] = gelu2(v[2 * i], v[2 * i + 1]);
      } else {
        __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        h[i] = *reinterpret_cast<uint32_t*>(&t);
      }
    }
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.out) + (long long)row0 * p.ld;
    if (p.pairs) {
      // an even lane stores its and the next lane's channel of row 2 i, the odd one of row 2 i + 1
      const bool odd = lane & 1;
      o += (odd ? p.ld : 0) + (ch & ~1);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, h[i], 1);
        const uint32_t w = odd ? __byte_perm(other, h[i], 0x7632) : __byte_perm(h[i], other, 0x5410);
        if (2 * i + (odd ? 1 : 0) < rows && ch < p.N) *reinterpret_cast<uint32_t*>(o) = w;
        o += 2 * p.ld;
      }
    } else if (ch < p.N) {
      o += ch;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const __nv_bfloat162 t = *reinterpret_cast<__nv_bfloat162*>(&h[i]);
        if (2 * i < rows) *o = t.x;
        o += p.ld;
        if (2 * i + 1 < rows) *o = t.y;
        o += p.ld;
      }
    }
  }
}

// PAIR: the CTAs of a cluster of two share an item (tcgen05 cta_group::2): 256 channels,
// 128 of them and half of the rows' codes in each one's shared memory. The first CTA's
// barriers take both CTAs' arrivals, its MMA lane issues for both.
//
// ROWS_M (bf16 output whose rows take 32-byte stores): the rows are the M operand and
// the channels N; otherwise the channels are M.
template <typename TO, bool GELU, int kStages, bool PAIR, bool ROWS_M>
__global__ void __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap tmM, const __grid_constant__ CUtensorMap tmN,
                   const __grid_constant__ CUtensorMap tmNM, const __grid_constant__ CUtensorMap tmNS,
                   const Params p) {
  constexpr uint32_t kStageBytes = stage_bytes(PAIR);
  constexpr int kCtas = PAIR ? 2 : 1, kM = 128 * kCtas, kRowTile = ROWS_M ? kM : kTN;
  const uint32_t rank = PAIR ? cluster_rank() : 0u;
  const bool leader = rank == 0;
  const int unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t s0 = smem_u32(smem);
  // stage s: weight codes, row codes
  auto stage = [&](int s) { return s0 + (uint32_t)s * kStageBytes; };
  uint8_t* scales = smem + kStages * kStageBytes;
  const uint32_t sc0 = smem_u32(scales);
  uint64_t* bars = reinterpret_cast<uint64_t*>(scales + kScaleBufs * kBytesS);
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto accf_bar = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
  auto acce_bar = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
  const uint32_t mma_done = bar0 + 8u * (2 * kStages + 4);
  auto sfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + 5 + b); };
  auto sempty_bar = [&](int b) { return bar0 + 8u * (2 * kStages + 5 + kScaleBufs + b); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  Item* list_s = reinterpret_cast<Item*>((reinterpret_cast<uintptr_t>(bars + kBars + 1) + 15) & ~(uintptr_t)15);
  int32_t* first_s = reinterpret_cast<int32_t*>(list_s + kListed);  // [G + 1] row tiles before each group
  int32_t* len_s = first_s + p.G + 1;                               // [G] rows of each group
  int32_t* start_s = len_s + p.G;                                   // [G] its first row

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(accf_bar(a), 1);
      mbar_init(acce_bar(a), kCtas * kEpiWarps);
    }
    for (int b = 0; b < kScaleBufs; ++b) {
      mbar_init(sfull_bar(b), kCtas * kScaleWarps);
      mbar_init(sempty_bar(b), 1);
    }
    mbar_init(mma_done, 1);
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
  // the warps' sums of rows and tiles, where the list of items comes later: no shared
  // memory beside that of smem_bytes
  long long* rows_sh = reinterpret_cast<long long*>(list_s);
  int* tiles_sh = reinterpret_cast<int*>(rows_sh + kThreads / 32);
  static_assert(kThreads / 32 * 12 <= kListed * sizeof(Item), "the list holds the warps' sums");
  grid_dep_wait();
  // Row tiles before each group; whatever the offsets hold, rows stay in [0, rows) and
  // the groups have no more than `rows` rows together.
  {
    long long rows_before = 0;
    int tiles_before = 0;
    for (int g0 = 0; g0 < p.G; g0 += kThreads) {
      const int g = g0 + (int)threadIdx.x;
      int n = 0, lo = 0;
      if (g < p.G) {
        lo = p.offsets ? min(max(p.offsets[g], 0), p.rows) : 0;
        n = max((p.offsets ? min(max(p.offsets[g + 1], 0), p.rows) : p.rows) - lo, 0);
      }
      long long upto = n;  // rows of the warp's groups up to this one
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
      }
      if (lane == 31) rows_sh[warp] = upto;
      __syncthreads();
      long long before = rows_before + upto - n;
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += rows_sh[w];
        rows_before += rows_sh[w];
      }
      n = (int)max(0ll, min((long long)n, p.rows - before));
      int tiles = (n + kRowTile - 1) / kRowTile, to = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, to, o);
        if (lane >= o) to += t;
      }
      if (lane == 31) tiles_sh[warp] = to;
      __syncthreads();
      int at = tiles_before + to - tiles;
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) at += tiles_sh[w];
        tiles_before += tiles_sh[w];
      }
      if (g < p.G) {
        first_s[g] = at;
        len_s[g] = n;
        start_s[g] = lo;
      }
    }
    if (threadIdx.x == 0) first_s[p.G] = tiles_before;
  }
  __syncthreads();
  const int ch_tiles = ROWS_M ? (p.N + kTN - 1) / kTN : (p.N + kM - 1) / kM;
  const int n_items = first_s[p.G] * ch_tiles;
  // `total` entries in `parts` equal parts, whole multiples of 16
  auto part_of = [](int total, int parts) { return ((total + parts - 1) / parts + 15) & ~15; };
  auto look_up = [&](int i) {
    const int tile = i / ch_tiles, ch = i - tile * ch_tiles;
    int lo = 0, hi = p.G - 1;  // the last group whose first tile is <= tile
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first_s[mid] <= tile) lo = mid; else hi = mid - 1;
    }
    const int k = tile - first_s[lo], rows = len_s[lo];
    Item it;
    int m, n;
    if (ROWS_M) {
      const int part = part_of(p.N, ch_tiles), at = k * kM + 128 * (int)rank;
      m = min(max(rows - at, 0), 128);
      it.m0 = start_s[lo] + min(at, rows);
      it.ch0 = ch * part;
      n = min(part, p.N - it.ch0);
      it.n0 = lo * p.N + it.ch0;
    } else {
      const int part = part_of(rows, first_s[lo + 1] - first_s[lo]);
      it.ch0 = ch * kM + 128 * (int)rank;
      m = min(max(p.N - it.ch0, 0), 128);
      it.m0 = lo * p.N + it.ch0;
      it.n0 = start_s[lo] + k * part;
      n = min(part, rows - k * part);
    }
    it.sizes = (uint32_t)m | (uint32_t)n << 16;
    return it;
  };
  for (int k = threadIdx.x; k < kListed; k += kThreads) {
    const long long i = unit + (long long)k * units;
    if (i < n_items) list_s[k] = look_up((int)i);
  }
  // the k-th item of this CTA (pair), i = unit + k units
  auto item_of = [&](int i, int k) { return k < kListed ? list_s[k] : look_up(i); };
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();  // both CTAs' barriers are set before either signals the other
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // Arrives at a barrier of the first CTA.
  auto arrive_leader = [&](uint32_t bar) {
    if (!PAIR || leader) mbar_arrive(bar);
    else mbar_arrive_cluster(mapa_shared(bar, 0));
  };
  auto commit = [&](uint32_t bar) {  // at this barrier of the pair's CTAs
    if (PAIR) umma_commit_pair(bar, 3);
    else umma_commit(bar);
  };

  if (warp < kEpiWarps) {
    // ---------------- accumulators to the output ----------------------------
    const int q = warp & 3, half = warp >> 2;
    int acc = 0;
    uint32_t ph = 0;
    for (int i = unit, k = 0; i < n_items; i += units, ++k) {
      const Item it = item_of(i, k);
      if (!wait_warp(accf_bar(acc), ph, abort_flag, p.status, p.wait_limit)) break;
      tc_fence_after();
      // (a quarter past the last entry of M has nothing to store)
      const int chunks = q * 32 < it.m() ? (it.n() + 31) / 32 : 0;
      const uint32_t from = tmem + acc * kAcc + ((uint32_t)(q * 32) << 16);
      float v[32];
      for (int c = half; c < chunks; c += 2) {
        tmem_ld32(from + c * 32, v);
        if (c + 2 >= chunks) {
          tc_fence_before();
          if (lane == 0) arrive_leader(acce_bar(acc));
        }
        if (ROWS_M) {
          if (q * 32 + lane < it.m())
            store_row<GELU>(p, v, it.m0 + q * 32 + lane, it.ch0 + c * 32, it.n() - c * 32);
        } else {
          store_chunk<TO, GELU>(p, v, it.n0 + c * 32, it.n() - c * 32, it.ch0 + q * 32 + lane, lane);
        }
      }
      if (half >= chunks && lane == 0) arrive_leader(acce_bar(acc));
      if (++acc == 2) { acc = 0; ph ^= 1u; }
    }
  } else if (warp == kTmaWarp) {
    // ---------------- codes of both operands --------------------------------
    // (One elected lane runs this role and the next from end to end: a branch for
    // one lane inside the loop costs the warp about 300 cycles to reconverge at every step, and
    // instructions under one lane's predicate are issued several times slower.)
    if (elect_one()) {
      bool ok = true;
      int s = 0;
      uint32_t ph = 0;
      long long issued = 0;
      for (int i = unit, k = 0; i < n_items && ok; i += units, ++k) {
        const Item it = item_of(i, k);
        // this CTA's entries of N
        const int n = PAIR ? ((it.n() + 15) & ~15) / 2 : it.n(), n0 = it.n0 + (int)rank * n;
        constexpr int kNM = kBoxM / kCtas, kNS = kBoxS / kCtas;
        const bool large = n > 2 * kNM, small = n <= kNS, two = !large && n > kNM;
        const CUtensorMap* map = large ? &tmN : small ? &tmNS : &tmNM;
        const uint32_t bytes =
            kBytesW + 128u * (uint32_t)(large ? stage_rows(PAIR) : small ? kNS : two ? 2 * kNM : kNM);
        auto load = [&](uint32_t dst, const CUtensorMap* from, uint32_t bar, int c0, int c1) {
          if (PAIR) tma_load_2d_pair(dst, from, mapa_shared(bar, 0), c0, c1);
          else tma_load_2d(dst, from, bar, c0, c1);
        };
        for (int kb = 0; kb < p.num_kb; ++kb) {
          ok = wait_bounded(empty_bar(s), ph ^ 1u, abort_flag, p.status, p.wait_limit);
          if (!ok) break;
          const uint32_t bar = full_bar(s);
          if (leader) mbar_expect_tx(bar, kCtas * bytes);
          load(stage(s), &tmM, bar, kb * 64, it.m0);
          load(stage(s) + kBytesW, map, bar, kb * 64, n0);
          if (two) load(stage(s) + kBytesW + kNM * 128u, map, bar, kb * 64, n0 + kNM);
          ++issued;
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
      // loads still in flight land before the CTA (pair) exits
      for (long long j = issued > kStages ? issued - kStages : 0; leader && j < issued; ++j)
        wait_settle(full_bar((int)(j % kStages)), (uint32_t)((j / kStages) & 1), p.wait_limit / 16);
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------- scales to TMEM, MMAs (the first CTA) ------------------
    if (leader && elect_one()) {
      int s = 0, acc = 0;
      uint32_t ph = 0, acc_ph = 0;
      int sb = 0;  // scale buffer and its phase
      uint32_t sb_ph = 0;
      bool ok = true, any = false;
      for (int i = unit, k = 0; i < n_items && ok; i += units, ++k) {
        const Item it = item_of(i, k);
        ok = wait_bounded(acce_bar(acc), acc_ph ^ 1u, abort_flag, p.status, p.wait_limit);
        if (!ok) break;
        tc_fence_after();
        const int n = (it.n() + 15) & ~15;
        const uint32_t d = tmem + acc * kAcc;
        const uint32_t id0 = idesc_mxf4(PAIR, n, 0), id2 = idesc_mxf4(PAIR, n, 2);
        // One step; h: its half of the scale buffer.
        auto step = [&](const int kb, const uint32_t h) {
          if (!wait_bounded(full_bar(s), ph, abort_flag, p.status, p.wait_limit)) return false;
          tc_fence_after();
          const uint32_t sc = sc0 + sb * kBytesS + h * 1024u;
          const uint32_t tw = tmem + kScaleCol + s * kScaleCols, ta = tw + 8;
          const uint64_t dw = scale_desc(sc), da = scale_desc(sc + kBytesSW + h * 1024u);
          copy_scales<PAIR>(tw, dw);
          copy_scales<PAIR>(tw + 4, dw + (512 >> 4));
          copy_scales<PAIR>(ta, da);
          copy_scales<PAIR>(ta + 8, da + (1024 >> 4));
          if (n > 128) {
            copy_scales<PAIR>(ta + 4, da + (512 >> 4));
            copy_scales<PAIR>(ta + 12, da + (1536 >> 4));
          }
          const uint64_t w = sw128_desc(stage(s)), a = sw128_desc(stage(s) + kBytesW);
          // 64 columns (32 bytes, two scales) at a time
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_mxf4<PAIR>(d, w + 2 * k, a + 2 * k, (k & 1) ? id2 : id0, tw + 4 * (k >> 1),
                     ta + 8 * (k >> 1), (kb | k) != 0 ? 1u : 0u);
          commit(empty_bar(s));
          any = true;
          if (++s == kStages) { s = 0; ph ^= 1u; }
          return true;
        };
        for (int kb = 0; kb < p.num_kb; kb += 2) {
          ok = wait_bounded(sfull_bar(sb), sb_ph, abort_flag, p.status, p.wait_limit) && step(kb, 0);
          if (ok && kb + 1 < p.num_kb) ok = step(kb + 1, 1);
          if (!ok) break;
          commit(sempty_bar(sb));
          if (++sb == kScaleBufs) { sb = 0; sb_ph ^= 1u; }
        }
        if (ok) commit(accf_bar(acc));
        if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
      }
      // every MMA issued has completed before TMEM is released
      if (any) {
        if (PAIR) umma_commit_pair(mma_done, 1);
        else umma_commit(mma_done);
        wait_settle(mma_done, 0u, p.wait_limit);
      }
    }
    __syncwarp();
  } else {
    // ---------------- scales ------------------------------------------------
    // Two steps at a time, two threads a row with eight bytes (a step's scales) each:
    // with a lane per row and step, every load touched 32 lines and the L1's tags were
    // taken 320 cycles a step.
    const int t = threadIdx.x - 32 * kScaleWarp, r0 = t >> 1, h = t & 1;
    int sb = 0;
    uint32_t sb_ph = 0;
    bool ok = true;
    for (int i = unit, k = 0; i < n_items && ok; i += units, ++k) {
      const Item it = item_of(i, k);
      const uint8_t* ws = p.m_scales + ((long long)it.m0 + r0) * p.pitch + 8 * h;
      const uint8_t* as = p.n_scales + ((long long)it.n0 + r0) * p.pitch + 8 * h;
      for (int kb = 0; kb < p.num_kb; kb += 2) {
        const bool in = kb + h < p.num_kb;
        uint2 w[2], a[3];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          w[r] = make_uint2(0u, 0u);
          if (in && 64 * r + r0 < it.m())
            w[r] = __ldg(reinterpret_cast<const uint2*>(ws + (long long)(64 * r) * p.pitch + kb * 8));
        }
#pragma unroll
        for (int r = 0; r < 3; ++r) {
          a[r] = make_uint2(0u, 0u);
          if (in && 64 * r + r0 < it.n())
            a[r] = __ldg(reinterpret_cast<const uint2*>(as + (long long)(64 * r) * p.pitch + kb * 8));
        }
        ok = wait_warp(sempty_bar(sb), sb_ph ^ 1u, abort_flag, p.status, p.wait_limit);
        if (!ok) break;
        // block of (step, 128 columns): byte 16 (row % 32) + 4 (row / 32)
        uint8_t* at = scales + sb * kBytesS + (r0 & 31) * 16 + h * 1024;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          uint32_t* to = reinterpret_cast<uint32_t*>(at + ((64 * r + r0) >> 5) * 4);
          to[0] = w[r].x;
          to[128] = w[r].y;
        }
        at += kBytesSW + h * 1024;
#pragma unroll
        for (int r = 0; r < 3; ++r) {
          uint32_t* to =
              reinterpret_cast<uint32_t*>(at + (r >> 1) * 512 + (((64 * r + r0) & 127) >> 5) * 4);
          to[0] = a[r].x;
          to[256] = a[r].y;
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) arrive_leader(sfull_bar(sb));
        if (++sb == kScaleBufs) { sb = 0; sb_ph ^= 1u; }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (PAIR) cluster_sync_all();
  if (warp == kMmaWarp) {
    if (PAIR) tmem_dealloc_pair(tmem, kTmemCols);
    else tmem_dealloc(tmem, kTmemCols);
  }
}

template <typename TO, bool GELU, int kStages, bool PAIR, bool ROWS_M>
cudaError_t launch_as(const CUtensorMap& tmM, const CUtensorMap (&tmN)[3], const Params& p, int grid,
                      cudaStream_t s) {
  const uint32_t smem = smem_bytes(PAIR, kStages, p.G);
  cudaError_t e = allow_smem_once(product_kernel<TO, GELU, kStages, PAIR, ROWS_M>, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = PAIR ? 2 : 1;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_kernel<TO, GELU, kStages, PAIR, ROWS_M>, tmM, tmN[0], tmN[1],
                            tmN[2], p);
}

template <typename TO, bool GELU>
cudaError_t launch(const CUtensorMap& tmM, const CUtensorMap (&tmN)[3], const Params& p, bool pair,
                   bool rows_m, int grid, cudaStream_t s) {
  if (pair) return launch_as<TO, GELU, kMaxStages, true, false>(tmM, tmN, p, grid, s);
  if (smem_bytes(false, kMaxStages, p.G) > kSmemMax)
    return launch_as<TO, GELU, kFewStages, false, false>(tmM, tmN, p, grid, s);
  if constexpr (sizeof(TO) == 2)
    if (rows_m) return launch_as<TO, GELU, kMaxStages, false, true>(tmM, tmN, p, grid, s);
  return launch_as<TO, GELU, kMaxStages, false, false>(tmM, tmN, p, grid, s);
}

}  // namespace fp4p
}  // namespace unif

using unif::set_error;
namespace fpp = unif::fp4p;

extern "C" {

int unif_moe_mxfp4_product(const uint8_t* a_codes, const uint8_t* a_scales, int64_t rows, int cols,
                           const uint8_t* w_codes, const uint8_t* w_scales, int n, int groups,
                           const int32_t* offsets, int activation, void* out, unif_moe_dtype dtype,
                           int64_t ld, int32_t* status, void* stream) {
  set_error("%s", "");
  if (rows < 0 || rows > 0x7fffffff - 1024 || n < 1 || groups < 1 || cols < 1 ||
      cols > UNIF_MOE_MXFP4_MAX_COLS || (int64_t)n * groups > 0x7fffffff - 1024) {
    set_error("bad sizes: rows=%lld cols=%d n=%d groups=%d", (long long)rows, cols, n, groups);
    return UNIF_MOE_ERR_ARG;
  }
  if (groups > UNIF_MOE_MXFP4_MAX_GROUPS) {
    set_error("groups=%d above %d", groups, UNIF_MOE_MXFP4_MAX_GROUPS);
    return UNIF_MOE_ERR_SHAPE;
  }
  if ((dtype != UNIF_MOE_F32 && dtype != UNIF_MOE_BF16) || activation < 0 ||
      activation > UNIF_MOE_ACTIVATION_GELU) {
    set_error("bad dtype %d or activation %d", (int)dtype, activation);
    return UNIF_MOE_ERR_ARG;
  }
  if (rows == 0) return UNIF_MOE_OK;
  if (!a_codes || !a_scales || !w_codes || !w_scales || !out || !status || (groups > 1 && !offsets)) {
    set_error("codes, scales, offsets, out or status is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  const uintptr_t codes = reinterpret_cast<uintptr_t>(a_codes) | reinterpret_cast<uintptr_t>(w_codes);
  const uintptr_t scales = reinterpret_cast<uintptr_t>(a_scales) | reinterpret_cast<uintptr_t>(w_scales);
  if ((codes & 15u) || (scales & 7u)) {
    set_error("codes must be 16-byte aligned, scales 8-byte");
    return UNIF_MOE_ERR_ARG;
  }
  if (ld < n) {
    set_error("the output's row stride %lld is below n=%d", (long long)ld, n);
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rc = unif::sm_count(&sms);
  if (rc != UNIF_MOE_OK) return rc;
  const uint64_t pitch = (uint64_t)(cols + 31) / 32 * 16;
  const bool fits = fpp::smem_bytes(false, fpp::kMaxStages, groups) <= fpp::kSmemMax;
  // Rows as M where tiles of 128 channels would waste a quarter of their work, groups
  // have rows enough, and the output takes 32-byte stores (us, channels as M and rows
  // as M, bf16 output with GELU and without: 100,003 rows in 272 groups of 192 x 768 29.8 and 23.2,
  // 22.4 and 22.2; 17,408 rows, 64 a group, 14.5 and 12.7, 11.6 and 11.4; 8,000 rows 11.3 and
  // 12.0, 10.3 and 9.7; 20,000 rows in 33 groups of 160 x 512 9.9 and 8.9, 7.3 and 7.1;
  // without waste, 60,000 rows in 33 groups of 384 x 1,536 27.6 and 28.6, 24.1 and 27.7, 100,000 of
  // 768 x 768 64.0 and 56.7, 44.2 and 56.0. fp32 output, when it had that form: 60,000 of 1,536 x
  // 384 66.6 and 86.9; rows off 32 bytes: 50,000 of 100 x 500 8.7 and 51.9).
  const bool wide = reinterpret_cast<uintptr_t>(out) % 32 == 0 && ld * (dtype == UNIF_MOE_F32 ? 4 : 2) % 32 == 0;
  const int parts = (n + fpp::kTN - 1) / fpp::kTN, part = ((n + parts - 1) / parts + 15) / 16 * 16;
  const int padded = (n + 127) / 128 * 128;
  const bool rows_m = fits && dtype == UNIF_MOE_BF16 && wide && 3ll * padded >= 4ll * parts * part &&
                      rows >= 64ll * groups;
  // CTA pairs, which read half of the rows' codes each, where steps are many enough for
  // operand traffic to bound the tile and a pair's 256 channels are no more
  // than two CTAs' 128 (us, single CTAs and pairs, bf16 output and fp32, 33 groups: 131,072
  // rows of 1,024 x 4,096 243 and 204, 270 and 237; 20,000 rows 50.2 and 45.9, 52.9 and 48.8;
  // 2,000 rows 18.1 and 18.6, 19.1 and 19.2; 500 rows 15.9 and 17.1, 16.2 and 17.1; 100,000 rows
  // of 1,024 x 1,024 63.0 and 60.7, 82.9 and 80.4; of 768 x 768 44.2 and 43.8, 59.1 and 59.3;
  // 1,000 rows of 4,096 x 1,024 in 8 groups 9.1 and 10.0, 10.1 and 10.8).
  const bool pair = fits && !rows_m && (n + 255) / 256 * 256 == padded && rows >= 32ll * groups &&
                    (cols >= 2048 || (cols >= 1024 && rows >= 1024ll * groups));
  const int ctas = pair ? 2 : 1;
  // 128-byte pieces of code rows, counted in 2-byte units
  const uint8_t* const m_codes = rows_m ? a_codes : w_codes;
  const uint8_t* const n_codes = rows_m ? w_codes : a_codes;
  const uint64_t w_rows = (uint64_t)n * groups, m_rows = rows_m ? (uint64_t)rows : w_rows,
                 n_rows = rows_m ? w_rows : (uint64_t)rows;
  CUtensorMap tmM, tmN[3];
  if (!unif::encode_bf16_map(&tmM, m_codes, pitch / 2, m_rows, 64, 128, 128) ||
      !unif::encode_bf16_map(&tmN[0], n_codes, pitch / 2, n_rows, 64, fpp::stage_rows(pair), 128) ||
      !unif::encode_bf16_map(&tmN[1], n_codes, pitch / 2, n_rows, 64, fpp::kBoxM / ctas, 128) ||
      !unif::encode_bf16_map(&tmN[2], n_codes, pitch / 2, n_rows, 64, fpp::kBoxS / ctas, 128)) {
    set_error("cuTensorMapEncodeTiled failed for the codes");
    return UNIF_MOE_ERR_CUDA;
  }
  fpp::Params p{};
  p.rows = (int)rows; p.N = n; p.G = groups;
  p.num_kb = (cols + fpp::kStep - 1) / fpp::kStep;
  const int ch_tile = rows_m ? fpp::kTN : 128 * ctas, row_tile = rows_m ? 128 * ctas : fpp::kTN;
  const int ch_tiles = (n + ch_tile - 1) / ch_tile;
  p.offsets = offsets;
  p.m_scales = rows_m ? a_scales : w_scales;
  p.n_scales = rows_m ? w_scales : a_scales;
  p.pitch = (cols + 255) / 256 * 8;
  p.out = out; p.ld = ld;
  p.pairs = (reinterpret_cast<uintptr_t>(out) & 3u) == 0 && ld % 2 == 0 && n % 2 == 0;
  p.status = status;
  p.wait_limit = unif::gemm_wait_limit();
  // at most one part-filled row tile per group beside the full ones
  const int64_t most = ((int64_t)rows / row_tile + (groups < rows ? groups : rows)) * ch_tiles;
  if (most > 0x7fff0000) {  // items are counted in 32 bits, beyond the last one by a grid
    set_error("too many tiles: rows=%lld n=%d groups=%d", (long long)rows, n, groups);
    return UNIF_MOE_ERR_SHAPE;
  }
  const int grid = ctas * (int)(most < sms / ctas ? most : sms / ctas);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  const bool gelu = activation == UNIF_MOE_ACTIVATION_GELU;
  if (dtype == UNIF_MOE_F32)
    e = gelu ? fpp::launch<float, true>(tmM, tmN, p, pair, rows_m, grid, s) : fpp::launch<float, false>(tmM, tmN, p, pair, rows_m, grid, s);
  else
    e = gelu ? fpp::launch<__nv_bfloat16, true>(tmM, tmN, p, pair, rows_m, grid, s)
             : fpp::launch<__nv_bfloat16, false>(tmM, tmN, p, pair, rows_m, grid, s);
  if (e != cudaSuccess) {
    set_error("mxfp4 product: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

}  // extern "C"

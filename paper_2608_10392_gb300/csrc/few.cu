// The whole layer for a few tokens (unif_moe_few_forward, unif_moe_forward_few): decisions,
// h = w GeLU(x K_e[:, H_b]) and y = sum h V_e[H_b, :] over the (expert, block) pairs that some
// token runs, in two kernels (three above 8 tokens).
//
// Bound by the weights' bytes: those of a pair are read once, whichever and however many tokens
// run it, and nothing else is large. No tiles of 128 rows are laid out for a token or two, no
// group table, no fp32 accumulator and no atomics: results repeat bit for bit.
//
// - up_kernel: every CTA takes the tokens' decisions for itself (up to 8 tokens; more are
//   decided by route_kernel, a CTA a token), lists the pairs in use, and its warps take tiles of
//   16 keys of a pair. The tokens of a pair are gathered: columns of the product are those that run it.
// - down_kernel: a cluster of CTAs takes 16 output features, its warps the pairs in turn, or 64 channels
//   of them where pairs are few. Columns are again a pair's tokens; a warp adds them to its sums of
//   all tokens in shared memory. The warps' sums meet there, the CTAs' in the cluster's, in a fixed
//   order.
//
// Weights stream through a ring of a warp's own in shared memory (cp.async, 2 KB a stage), so that what
// is on its way does not depend on registers; the products are mma.sync, a thread's 32 bytes of a row
// standing for other positions than the fragment's, the same ones for both operands, which a sum
// does not notice. (24 tokens of the 33-expert layer of 1,024 / 4,096, 272 MB of weights in each kernel: 53 and 75 us;
// weights straight into registers 67 and 118.) One token takes 16 us (launches, decisions, the drain of two
// kernels) and the time of its pairs' bytes, 1.05 MB each: 16 pairs 18.8 us (floor 2.5), 48 23.1 (7.4), 80 26.9 (12.4), 168
// 42.4 (25.9); the forward 75. 8 tokens take 72 to 83 us, 16 105, 24 129, 64 152, the forward 133, 153, 151 and 154.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "gelu_log.cuh"
#include "internal.cuh"
#include "overlap.h"

namespace unif {
namespace few {

constexpr int kThreads = 256, kWarps = kThreads / 32;  // of route_kernel and down_kernel
constexpr int kUpWarps = 16;  // one CTA an SM: fewer read the router
constexpr int kMost = UNIF_MOE_FEW_TOKENS;
constexpr size_t kSmemMost = 232448;
constexpr int kTogether = 8;  // most tokens that every CTA decides for itself

struct Params {
  int T, d, H, K, B, M, C;        // C = 1 + K + B: rows of the router
  float tau, alpha_fixed, beta_fixed;
  int topk_fixed, prefix;
  const __nv_bfloat16* x;
  long long ld_x;
  const __nv_bfloat16* router;    // [C][d]
  const float* bias;              // [K + 1] or NULL
  const __nv_bfloat16 *up, *down; // [K + 1][H][d], [K + 1][d][H]
  const uint8_t* mask;
  __nv_bfloat16* out;
  long long ld_out;
  int32_t *b_out, *k_out;
  // workspace
  uint64_t *shr, *em;             // [T] blocks of the shared expert, residual experts
  float* alpha;                   // [T]
  float* s;                       // [T][K] affinities
  int* n_pairs;                   // pairs in use, in the order of (expert, block)
  uint16_t* pair;                 // [G], as pair_code
  uint64_t* members;              // [B + K] tokens whose shared set has a block, that take an expert
  __nv_bfloat16* h;               // [K + 1][T][H], of the pairs' tokens
};

// A pair as it is listed, expert and block without a division.
__device__ __forceinline__ uint16_t pair_code(int e, int b) { return (uint16_t)(e << 6 | b); }
__device__ __forceinline__ int expert_of(int code) { return code >> 6; }
__device__ __forceinline__ int block_of(int code) { return code & 63; }

// Every `step`-th of the (pair, part) items, `parts` to a pair, without a division for each.
struct Walk {
  int pair, part;
  int by_pair, by_part, parts;
  __device__ __forceinline__ Walk(int first, int step, int parts_) : parts(parts_) {
    pair = first / parts_;
    part = first - pair * parts_;
    by_pair = step / parts_;
    by_part = step - by_pair * parts_;
  }
  __device__ __forceinline__ void next() {
    pair += by_pair;
    part += by_part;
    if (part >= parts) {
      part -= parts;
      ++pair;
    }
  }
};

// Thirty-two bytes: sixteen bf16 values as eight operand registers.
struct Piece {
  uint32_t r[8];
};
__device__ __forceinline__ void clear(Piece& p) {
#pragma unroll
  for (int i = 0; i < 8; ++i) p.r[i] = 0u;
}
// A warp's ring of weights: stages of 16 rows by 128 bytes, 16 bytes of a row at the place that the
// row's number mixes (so that fragments are read without bank conflicts).
constexpr uint32_t kStage = 2048;
template <int S>
struct Ring {
  uint32_t base;
  int lane, put = 0, get = 0;
  __device__ __forceinline__ Ring(uint32_t base_, int lane_) : base(base_), lane(lane_) {}
  // 16 rows `ld` elements apart from `from` on, on their way to the next stage (nothing where `on` is
  // false); the stage read last must not be in use any more
  __device__ __forceinline__ void fetch(bool on, const __nv_bfloat16* from, long long ld) {
    __syncwarp();
    if (on) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (lane >> 3) + 4 * i, piece = lane & 7;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + put * kStage + row * 128 +
                                                                      ((piece ^ (row & 7)) << 4)),
                     "l"(from + row * ld + piece * 8)
                     : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    put = put + 1 == S ? 0 : put + 1;
  }
  // The oldest stage's fragments: rows g and g + 8 of this thread.
  __device__ __forceinline__ void read(Piece& lo, Piece& hi) {
    asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
    __syncwarp();
    const int g = lane >> 2, c = (lane & 3) * 2;
    const uint32_t row = base + get * kStage + g * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = row + (((c + h) ^ g) << 4);
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(lo.r[4 * h]), "=r"(lo.r[4 * h + 1]), "=r"(lo.r[4 * h + 2]), "=r"(lo.r[4 * h + 3])
                   : "r"(at)
                   : "memory");
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(hi.r[4 * h]), "=r"(hi.r[4 * h + 1]), "=r"(hi.r[4 * h + 2]), "=r"(hi.r[4 * h + 3])
                   : "r"(at + 1024)
                   : "memory");
    }
    get = get + 1 == S ? 0 : get + 1;
  }
};
// Tokens (16-byte aligned).
__device__ __forceinline__ void read_token(Piece& p, const __nv_bfloat16* from) {
  const uint4 a = *reinterpret_cast<const uint4*>(from), b = *(reinterpret_cast<const uint4*>(from) + 1);
  p.r[0] = a.x; p.r[1] = a.y; p.r[2] = a.z; p.r[3] = a.w;
  p.r[4] = b.x; p.r[5] = b.y; p.r[6] = b.z; p.r[7] = b.w;
}
// c += rows (g: lo, g + 8: hi) x columns (token g) over 64 features of four threads.
__device__ __forceinline__ void multiply(float (&c)[4], const Piece& lo, const Piece& hi, const Piece& x) {
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
        " {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(lo.r[i]), "r"(hi.r[i]), "r"(lo.r[i + 1]), "r"(hi.r[i + 1]), "r"(x.r[i]), "r"(x.r[i + 1]));
}

// ---- decisions ----

// Those of token t by one warp, from its row z of the router's product (Eqs. 18-27): the orders
// are ranks (larger first, ties to the lower index), as in decide.cuh. Each lane holds
// entries lane and lane + 32 of the experts and of the blocks.
__device__ __forceinline__ void decide(const Params& p, int t, bool valid, const float* z, int lane, uint64_t& shr,
                                       uint64_t& em, float& alpha, float* s, int& count, int& taken) {
  const int K = p.K, B = p.B;
  shr = em = 0ull;
  alpha = 0.f;
  count = taken = 0;
  float l[2], e[2], u[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = lane + 32 * i;
    l[i] = valid && j < K ? z[1 + j] + (p.bias ? p.bias[1 + j] : 0.f) : -INFINITY;
    u[i] = valid && j < B ? z[1 + K + j] : -INFINITY;
  }
  if (valid) {
    float most = fmaxf(l[0], l[1]);
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float den = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e[i] = lane + 32 * i < K ? expf(l[i] - most) : 0.f;
      den += e[i];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
    const float z0 = z[0] + (p.bias ? p.bias[0] : 0.f);
    alpha = isnan(p.alpha_fixed) ? p.tau + (1.f - 2.f * p.tau) * (1.f / (1.f + expf(-z0))) : p.alpha_fixed;
    count = min(max(__float2int_rn((float)B * alpha), 0), B);
    const float inv = 1.f / den;
    e[0] *= inv;
    e[1] *= inv;
    // ranks of the blocks, ranks of the experts and the mass up to each
    int rb[2] = {0, 0}, re[2] = {0, 0};
    float mass[2] = {0.f, 0.f};
#pragma unroll 8
    for (int i = 0; i < (p.prefix ? 0 : B); ++i) {
      const float v = __shfl_sync(0xffffffffu, i < 32 ? u[0] : u[1], i & 31);
#pragma unroll
      for (int k = 0; k < 2; ++k) rb[k] += v > u[k] || (v == u[k] && i < lane + 32 * k);
    }
#pragma unroll 8
    for (int i = 0; i < K; ++i) {
      const float v = __shfl_sync(0xffffffffu, i < 32 ? l[0] : l[1], i & 31);
      const float w = __shfl_sync(0xffffffffu, i < 32 ? e[0] : e[1], i & 31);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int j = lane + 32 * k;
        const bool before = v > l[k] || (v == l[k] && i < j);
        re[k] += before;
        mass[k] += before || i == j ? w : 0.f;
      }
    }
    const float beta = isnan(p.beta_fixed) ? 1.f - alpha : p.beta_fixed;
    int k = K;  // (where rounding leaves every sum below beta)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (lane + 32 * i < K && mass[i] >= beta) k = min(k, re[i] + 1);
    taken = p.topk_fixed > 0 ? p.topk_fixed : __reduce_min_sync(0xffffffffu, k);
    uint32_t bits[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = lane + 32 * i;
      bits[i] = __ballot_sync(0xffffffffu, j < B && (p.prefix ? j : rb[i]) < count);
      bits[2 + i] = __ballot_sync(0xffffffffu, j < K && re[i] < taken);
      if (j < K) s[j] = e[i];
    }
    shr = (uint64_t)bits[1] << 32 | bits[0];
    em = (uint64_t)bits[3] << 32 | bits[2];
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (lane + 32 * i < K) s[lane + 32 * i] = 0.f;
  }
}

// Shared memory of the router's product: [warps][rows of the router, in 16s][8 tokens], then [8][C].
__host__ __device__ inline int router_rows(int C) { return (C + 15) / 16 * 16; }
__host__ __device__ inline int route_floats(int C, int warps) { return warps * router_rows(C) * 8 + 8 * C; }

// z [8][C] of the tokens from t0 on (up to 8): the CTA's warps share the features.
template <int WARPS>
__device__ __forceinline__ float* route_products(const Params& p, int t0, int count, float* sm) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, at = (lane & 3) * 16;
  const int R = router_rows(p.C);
  float* mine = sm + warp * R * 8;
  const bool there = g < count;
  const __nv_bfloat16* x = p.x + (long long)(t0 + (there ? g : 0)) * p.ld_x + at;
  for (int r0 = 0; r0 < R; r0 += 64) {  // four tiles of 16 rows at a time
    float c[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[k][i] = 0.f;
    for (int f = warp * 64; f < p.d; f += WARPS * 64) {
      Piece v, lo[4], hi[4];
      clear(v);
      if (there) read_token(v, x + f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r0 + 16 * k + g;
        clear(lo[k]);
        clear(hi[k]);
        if (r < p.C) read_token(lo[k], p.router + (long long)r * p.d + f + at);
        if (r + 8 < p.C) read_token(hi[k], p.router + (long long)(r + 8) * p.d + f + at);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) multiply(c[k], lo[k], hi[k], v);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r0 + 16 * k + g, n = (lane & 3) * 2;
      if (r0 + 16 * k >= R) continue;
      mine[r * 8 + n] = c[k][0];
      mine[r * 8 + n + 1] = c[k][1];
      mine[(r + 8) * 8 + n] = c[k][2];
      mine[(r + 8) * 8 + n + 1] = c[k][3];
    }
  }
  __syncthreads();
  float* z = sm + WARPS * R * 8;
  for (int i = threadIdx.x; i < 8 * p.C; i += WARPS * 32) {
    const int n = i & 7, r = i >> 3;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) v += sm[w * R * 8 + r * 8 + n];
    z[n * p.C + r] = v;
  }
  __syncthreads();
  return z;
}

// A token to a CTA (more than kTogether tokens).
__global__ void __launch_bounds__(kThreads) route_kernel(const Params p) {
  extern __shared__ float sm[];
  grid_dep_wait();
  grid_dep_launch();
  const int t = blockIdx.x;
  const bool valid = !p.mask || p.mask[t];
  const float* z = route_products<kWarps>(p, t, 1, sm);
  if (threadIdx.x >= 32) return;
  uint64_t shr, em;
  float alpha;
  int count, taken;
  const int lane = threadIdx.x;
  decide(p, t, valid, z, lane, shr, em, alpha, p.s + (long long)t * p.K, count, taken);
  if (lane == 0) {
    p.shr[t] = shr;
    p.em[t] = em;
    p.alpha[t] = alpha;
    if (p.b_out) p.b_out[t] = count;
    if (p.k_out) p.k_out[t] = taken;
  }
}

// ---- h ----

struct UpShared {
  uint64_t shr[kMost], em[kMost];
  uint64_t in_block[64], in_expert[64];  // tokens whose shared set has a block; that take an expert
  float alpha[kMost];
  int found[kUpWarps];
  uint8_t slots[kUpWarps][kMost];          // a warp's tokens of its pair
};
constexpr int kUpStages = 6;
// Tokens held in shared memory: rows of d values and 16 bytes.
__host__ __device__ inline size_t held_bytes(int T, int d) { return ((size_t)T * (2 * d + 16) + 127) / 128 * 128; }
// After it: the affinities [8][K] where the decisions are taken here, [G] pairs in use, then the rings
// (before they are in use, the router's product in their place).
__host__ __device__ inline size_t up_fixed(int G, int K, bool routes) {
  return ((sizeof(UpShared) + (size_t)G * 2 + (routes ? 32 * (size_t)K : 0)) + 127) / 128 * 128 + 128;
}
__host__ __device__ inline size_t up_smem(int G, int K, int C, bool routes, int stages, size_t held) {
  const size_t rings = (size_t)kUpWarps * stages * kStage + held, product = routes ? 4 * (size_t)route_floats(C, kUpWarps) : 0;
  return up_fixed(G, K, routes) + (rings > product ? rings : product);
}

// NT: pieces of eight tokens that are taken at once; a pair that more tokens run is gone through again.
// ROUTES: the decisions are taken here. HELD: the tokens are held in shared memory, in rings of that many stages
// (0: they come from L1, of which the rings leave little, so that up to half as many bytes again come from L2; the
// layer in us, without and with, 1,024 / 4,096, 33 experts: 24 tokens 139 and 129, 48 160 and 137, 64, two stages, 174
// and 152; 768 wide, 17 experts: 64 tokens, three stages, 84 and 71; up to 8 tokens there is nothing to gain).
template <int NT, bool ROUTES, int HELD>
__global__ void __launch_bounds__(32 * kUpWarps, 1) up_kernel(const Params p) {
  constexpr int S = HELD ? HELD : kUpStages;
  constexpr int kThreads = 32 * kUpWarps, kWarps = kUpWarps;
  extern __shared__ __align__(16) uint8_t raw[];
  UpShared& sh = *reinterpret_cast<UpShared*>(raw);
  const int G = (p.K + 1) * p.B;
  float* s = reinterpret_cast<float*>(raw + sizeof(UpShared));               // [8][K]
  uint16_t* list = reinterpret_cast<uint16_t*>(s + (ROUTES ? 8 * p.K : 0));  // [G]
  static_assert(sizeof(UpShared) % 8 == 0, "what follows is aligned");
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(raw));
  const uint32_t rings = (base + (uint32_t)up_fixed(G, p.K, ROUTES) - 1u) & ~127u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool first = blockIdx.x == 0;
  grid_dep_wait();
  grid_dep_launch();
  if constexpr (ROUTES) {
    const float* z = route_products<kUpWarps>(p, 0, p.T, reinterpret_cast<float*>(raw + (rings - base)));
    if (warp < p.T) {
      uint64_t shr, em;
      float alpha;
      int count, taken;
      decide(p, warp, !p.mask || p.mask[warp], z + warp * p.C, lane, shr, em, alpha, s + warp * p.K, count, taken);
      if (lane == 0) {
        sh.shr[warp] = shr;
        sh.em[warp] = em;
        sh.alpha[warp] = alpha;
        if (first) {
          if (p.b_out) p.b_out[warp] = count;
          if (p.k_out) p.k_out[warp] = taken;
        }
      }
    }
  } else {
    for (int t = threadIdx.x; t < p.T; t += kThreads) {
      sh.shr[t] = p.shr[t];
      sh.em[t] = p.em[t];
      sh.alpha[t] = p.alpha[t];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.B + p.K; i += kThreads) {
    uint64_t v = 0ull;
    for (int t = 0; t < p.T; ++t) v |= ((i < p.B ? sh.shr[t] >> i : sh.em[t] >> (i - p.B)) & 1ull) << t;
    if (i < p.B) sh.in_block[i] = v;
    else sh.in_expert[i - p.B] = v;
  }
  __syncthreads();
  auto members = [&](int code) {
    const int e = expert_of(code), b = block_of(code);
    return e == 0 ? sh.in_block[b] : sh.in_expert[e - 1] & ~sh.in_block[b];
  };
  // pairs in use, in order: a run of them to each thread
  const int each = (G + kThreads - 1) / kThreads, from = threadIdx.x * each, to = min(G, from + each);
  auto code_of = [&](int i) {
    const int e = i / p.B;
    return pair_code(e, i - e * p.B);
  };
  int n = 0;
  for (int i = from; i < to; ++i) n += members(code_of(i)) != 0ull;
  int before = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += t;
  }
  if (lane == 31) sh.found[warp] = before;
  __syncthreads();
  int to_at = before - n, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) to_at += sh.found[w];
    all += sh.found[w];
  }
  for (int i = from; i < to; ++i) {
    const uint16_t code = code_of(i);
    if (members(code) == 0ull) continue;
    list[to_at] = code;
    if (first) p.pair[to_at] = code;
    ++to_at;
  }
  if (first && threadIdx.x == 0) *p.n_pairs = all;
  __syncthreads();

  const uint32_t held = rings + kWarps * S * kStage, pitch = 2 * p.d + 16;
  if constexpr (HELD != 0) {
    const int pieces = p.d / 8;
    for (int i = threadIdx.x; i < p.T * pieces; i += kThreads) {
      const int t = i / pieces, c = i - t * pieces;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(held + t * pitch + c * 16),
                   "l"(p.x + (long long)t * p.ld_x + c * 8)
                   : "memory");
    }
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
    __syncthreads();
  }

  if (first)
    for (int i = threadIdx.x; i < p.B + p.K; i += kThreads)
      p.members[i] = i < p.B ? sh.in_block[i] : sh.in_expert[i - p.B];

  // tiles of 16 keys, in blocks of 64 features
  const int blocks = p.d / 64;
  const Walk begin((int)(warp * gridDim.x + blockIdx.x), (int)(gridDim.x * kWarps), p.M / 16);
  const int g = lane >> 2, k0 = (lane & 3) * 16;
  uint8_t* slots_all = sh.slots[warp];
  Ring<S> ring(rings + (uint32_t)warp * S * kStage, lane);
  Walk next = begin;          // of the blocks on their way
  int next_f = 0, again = 0;  // their features; times that the item's blocks are needed once more
  const __nv_bfloat16* keys = nullptr;
  auto enter = [&]() {
    if (next.pair >= all) return;
    const int code = list[next.pair];
    keys = p.up + ((long long)expert_of(code) * p.H + block_of(code) * p.M + next.part * 16) * p.d;
    again = p.T <= 8 * NT ? 0 : (__popcll(members(code)) - 1) / (8 * NT);
  };
  enter();
  auto fetch = [&]() {
    ring.fetch(next.pair < all, keys + next_f, p.d);
    if ((next_f += 64) == p.d) {
      next_f = 0;
      if (--again < 0) {
        next.next();
        enter();
      }
    }
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fetch();
  for (Walk at = begin; at.pair < all; at.next()) {
    const int code = list[at.pair], row = at.part * 16;
    const int e = expert_of(code), b = block_of(code);
    const uint64_t m = members(code);
    const int all_tokens = __popcll(m);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int t = lane + 32 * k;
      if (m >> t & 1ull) slots_all[__popcll(m & ((1ull << t) - 1ull))] = (uint8_t)t;
    }
    __syncwarp();
    for (int s0 = 0; s0 < all_tokens; s0 += 8 * NT) {
    const uint8_t* slots = slots_all + s0;
    const int tokens = min(all_tokens - s0, 8 * NT), pieces = (tokens + 7) / 8;
    const __nv_bfloat16* x[NT];
    uint32_t xs[NT];
    auto token = [&](Piece& v, int t, int f) {  // 64 features of piece t's tokens
      if constexpr (HELD != 0) {
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.r[0]), "=r"(v.r[1]), "=r"(v.r[2]), "=r"(v.r[3])
                     : "r"(xs[t] + 128 * f));
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.r[4]), "=r"(v.r[5]), "=r"(v.r[6]), "=r"(v.r[7])
                     : "r"(xs[t] + 128 * f + 16));
      } else {
        read_token(v, x[t] + 64 * f);
      }
    };
    float c[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int slot = t * 8 + g;
      const int tok = slot < tokens ? slots[slot] : slots[0];
      if constexpr (HELD != 0) xs[t] = held + tok * pitch + k0 * 2;
      else x[t] = p.x + (long long)tok * p.ld_x + k0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c[t][j] = 0.f;
    }
    Piece v;
    token(v, 0, 0);
    for (int f = 0; f < blocks; ++f) {
      Piece lo, hi;
      fetch();
      ring.read(lo, hi);
      multiply(c[0], lo, hi, v);
#pragma unroll
      for (int t = 1; t < NT; ++t)
        if (t < pieces) {
          token(v, t, f);
          multiply(c[t], lo, hi, v);
        }
      if (f + 1 < blocks) token(v, 0, f + 1);
    }
    // h = w GeLU, rounded once: the weight comes before the rounding, so that the down projection
    // adds up what is held
    __nv_bfloat16* h = p.h + (long long)e * p.T * p.H + b * p.M + row + g;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t >= pieces) continue;
      gelu::gelu2(c[t][0], c[t][1]);
      gelu::gelu2(c[t][2], c[t][3]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int slot = t * 8 + (lane & 3) * 2 + j;
        if (slot >= tokens) continue;
        const int tok = slots[slot];
        const float w = e == 0 ? sh.alpha[tok]
                               : ROUTES ? s[tok * p.K + e - 1] : __ldg(p.s + (long long)tok * p.K + e - 1);
        h[(long long)tok * p.H] = __float2bfloat16_rn(w * c[t][j]);
        h[(long long)tok * p.H + 8] = __float2bfloat16_rn(w * c[t][2 + j]);
      }
    }
    }
  }
}

// ---- y ----

// Stages such that two CTAs are on an SM. Shared memory: the masks, the pairs in use [G], the warps'
// sums [warps][TOK tokens][16], the CTA's, the rings.
__host__ __device__ constexpr int down_stages(int TOK) { return TOK <= 32 ? 5 : 4; }
template <int TOK>
constexpr size_t down_smem(int G) {
  return 128 * 8 + ((size_t)G * 2 + 15) / 16 * 16 + 4u * (kWarps + 1) * 16 * TOK + 128 +
         (size_t)kWarps * down_stages(TOK) * kStage;
}

// NT as in up_kernel; TOK: most tokens.
template <int NT, int TOK>
__global__ void __launch_bounds__(kThreads, 2) down_kernel(const Params p, const int ctas) {
  extern __shared__ __align__(16) uint8_t raw[];
  __shared__ uint8_t slots_of[kWarps][4][kMost];  // the tokens of the last four items
  constexpr int kSums = 16 * TOK, S = down_stages(TOK);
  const int G = (p.K + 1) * p.B;
  uint64_t* masks = reinterpret_cast<uint64_t*>(raw);
  uint16_t* list = reinterpret_cast<uint16_t*>(masks + 128);
  float* red = reinterpret_cast<float*>(raw + 128 * 8 + ((size_t)G * 2 + 15) / 16 * 16);
  const uint32_t rings = ((uint32_t)__cvta_generic_to_shared(red + (kWarps + 1) * kSums) + 127u) & ~127u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % ctas, j0 = blockIdx.x / ctas * 16;
  const int g = lane >> 2, k0 = (lane & 3) * 16;
  float* mine = red + warp * kSums;  // [token][feature]
  for (int i = lane; i < kSums; i += 32) mine[i] = 0.f;
  grid_dep_wait();
  const int pairs = *p.n_pairs;
  for (int i = threadIdx.x; i < p.B + p.K; i += kThreads) masks[i] = p.members[i];
  for (int i = threadIdx.x; i < pairs; i += kThreads) list[i] = p.pair[i];
  __syncthreads();
  // items: whole pairs where every warp of the cluster has several, else their chunks of 64 channels
  const int per = p.M / 64, units = ctas * kWarps;
  const int length = pairs >= 8 * units ? per : 1;
  const Walk begin(warp * ctas + rank, units, per / length);
  const __nv_bfloat16* rows = p.down + (long long)j0 * p.H;
  struct At {
    Walk w;
    int k, again, e, b, ch;  // chunk of the item, times that it is needed once more; expert, block, first
  };                         // channel of the chunk
  auto members = [&](const At& a) {
    return a.e == 0 ? masks[a.b] : masks[p.B + a.e - 1] & ~masks[a.b];
  };
  auto enter = [&](At& a) {
    const int code = list[a.w.pair];
    a.k = 0;
    a.e = expert_of(code);
    a.b = block_of(code);
    a.ch = a.b * p.M + a.w.part * length * 64;
    a.again = TOK <= 8 * NT ? 0 : (__popcll(members(a)) - 1) / (8 * NT);
  };
  At next{begin, 0, 0, 0, 0, 0};
  if (next.w.pair < pairs) enter(next);
  Ring<S> ring(rings + (uint32_t)warp * S * kStage, lane);
  auto fetch = [&]() {
    const bool on = next.w.pair < pairs;
    ring.fetch(on, rows + (long long)next.e * p.d * p.H + next.ch, p.H);
    if (!on) return;
    next.ch += 64;
    if (++next.k == length) {
      if (--next.again >= 0) {
        next.k = 0;
        next.ch -= 64 * length;
      } else {
        next.w.next();
        if (next.w.pair < pairs) enter(next);
      }
    }
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fetch();
  // A step: a chunk for up to 8 NT of its pair's tokens, or (up to 8 tokens) for all of them, with 0 for
  // those that do not run the pair. h of a step is read kAhead steps before it is used: its latency
  // is longer than a step (a step ahead: 0.9 us a step, 24 tokens of the 33-expert layer 69 us).
  constexpr bool kAll = TOK <= 8;
  constexpr int P = NT < 2 ? NT : 2;  // pieces of h that are read ahead
  constexpr int kAhead = kAll ? 4 : 2;
  struct Step {
    bool on, last;  // there is one; it is the last of its item's tokens
    int tokens;
    uint32_t taking;  // (kAll) the tokens that run the pair
    const uint8_t* slots;
    const __nv_bfloat16* h;
  };
  At ahead{begin, 0, 0, 0, 0, 0};
  int all_tokens = 0, s0 = 0, turn = 0;
  uint64_t taking = 0ull;  // the item's tokens
  auto open = [&]() {  // the item that `ahead` is at: its tokens, listed
    if (ahead.w.pair >= pairs) return;
    enter(ahead);
    taking = members(ahead);
    if constexpr (kAll) {
      all_tokens = p.T;
    } else {
      turn = (turn + 1) & 3;
      uint8_t* to = slots_of[warp][turn];
#pragma unroll
      for (int k = 0; k < (TOK + 31) / 32; ++k) {
        const int t = lane + 32 * k;
        if (taking >> t & 1ull) to[__popcll(taking & ((1ull << t) - 1ull))] = (uint8_t)t;
      }
      __syncwarp();
      all_tokens = __popcll(taking);
    }
  };
  Piece v[kAhead][P];
  auto take = [&](Piece (&to)[P]) {  // the next step, its h on its way
    Step st{ahead.w.pair < pairs, false, 0, (uint32_t)taking, nullptr, nullptr};
    if (!st.on) return st;
    st.h = p.h + (long long)ahead.e * p.T * p.H + ahead.ch + k0;
    if constexpr (kAll) {
      clear(to[0]);
      if (taking >> g & 1ull) read_token(to[0], st.h + (long long)g * p.H);
    } else {
      st.slots = slots_of[warp][turn] + s0;
      st.tokens = min(all_tokens - s0, 8 * NT);
#pragma unroll
      for (int t = 0; t < P; ++t)
        if (t * 8 < st.tokens) {
          const int slot = t * 8 + g;  // (columns past the tokens repeat the first one)
          read_token(to[t], st.h + (long long)st.slots[slot < st.tokens ? slot : 0] * p.H);
        }
    }
    if (++ahead.k < length) {
      ahead.ch += 64;
    } else {
      st.last = true;
      ahead.k = 0;
      ahead.ch -= 64 * (length - 1);
      s0 += 8 * NT;
      if (kAll || s0 >= all_tokens) {
        s0 = 0;
        ahead.w.next();
        open();
      }
    }
    return st;
  };
  float c[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) c[t][j] = 0.f;
  open();
  Step steps[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) steps[k] = take(v[k]);
  while (steps[0].on) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const Step now = steps[k];
      if (!now.on) {  // the last step was the one before
        steps[0].on = false;
        break;
      }
      Piece lo, hi;
      fetch();
      ring.read(lo, hi);
      if constexpr (kAll) {
        // (what does not run the pair adds nothing of it, not 0 times an infinity either)
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        multiply(y, lo, hi, v[k][0]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (now.taking >> ((lane & 3) * 2 + (j & 1)) & 1u) c[0][j] += y[j];
      } else {
#pragma unroll
        for (int t = 0; t < NT; ++t)
          if (t * 8 < now.tokens) {
            if (t < P) {
              multiply(c[t], lo, hi, v[k][t < P ? t : 0]);
            } else {
              Piece w;
              const int slot = t * 8 + g;
              read_token(w, now.h + (long long)now.slots[slot < now.tokens ? slot : 0] * p.H);
              multiply(c[t], lo, hi, w);
            }
          }
        if (now.last) {  // the columns to their tokens
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int slot = t * 8 + (lane & 3) * 2 + (j & 1);
              if (slot < now.tokens) mine[now.slots[slot] * 16 + g + (j >> 1) * 8] += c[t][j];
              c[t][j] = 0.f;
            }
        }
      }
      steps[k] = take(v[k]);
    }
  }
  if constexpr (kAll)
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[((lane & 3) * 2 + (j & 1)) * 16 + g + (j >> 1) * 8] = c[0][j];
  __syncthreads();
  float* sums = red + kWarps * kSums;
  for (int i = threadIdx.x; i < kSums; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += red[w * kSums + i];
    sums[i] = v;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  // each CTA adds a share of the cluster's sums
  const uint32_t here = static_cast<uint32_t>(__cvta_generic_to_shared(sums));
  for (int i = rank * kThreads + threadIdx.x; i < 16 * p.T; i += ctas * kThreads) {
    float v = 0.f;
    for (int r = 0; r < ctas; ++r) {
      uint32_t there;
      float a;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here + 4u * i), "r"(r));
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(a) : "r"(there) : "memory");
      v += a;
    }
    p.out[(i >> 4) * p.ld_out + j0 + (i & 15)] = __float2bfloat16_rn(v);
  }
  // no CTA leaves while another reads its sums
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- the router's rows ----

// Row c of [1 + K + B][d]: column c of w_router [d][K + 1], or the mean key of block c - K - 1 of the
// shared expert, summed in fp64 and rounded once.
__global__ void __launch_bounds__(256)
    table_kernel(int d, int K, int B, int M, const __nv_bfloat16* w_router, const __nv_bfloat16* up,
                 __nv_bfloat16* table) {
  grid_dep_wait();
  const int i = blockIdx.x * 256 + threadIdx.x, c = blockIdx.y;
  if (i >= d) return;
  if (c <= K) {
    table[(long long)c * d + i] = w_router[(long long)i * (K + 1) + c];
    return;
  }
  double sum = 0.0;
  const __nv_bfloat16* key = up + (long long)(c - K - 1) * M * d + i;
  for (int h = 0; h < M; ++h) sum += (double)__bfloat162float(key[(long long)h * d]);
  const double mean = sum / (double)M;
  // towards zero with the last bit set where that was not exact: the second rounding is then right
  float f = __double2float_rz(mean);
  if ((double)f != mean) f = __uint_as_float(__float_as_uint(f) | 1u);
  table[(long long)c * d + i] = __float2bfloat16_rn(f);
}

// ---- host side ----

int check(const unif_moe_few* p) {
  if (!p) { set_error("the description is NULL"); return UNIF_MOE_ERR_ARG; }
  if (p->tokens < 0 || p->d_model < 1 || p->d_ff < 1 || p->n_experts < 1 || p->n_experts > 64 || p->n_blocks < 2 ||
      p->n_blocks > 64) {
    set_error("bad sizes: tokens=%d d_model=%d d_ff=%d n_experts=%d n_blocks=%d", p->tokens, p->d_model, p->d_ff,
              p->n_experts, p->n_blocks);
    return UNIF_MOE_ERR_ARG;
  }
  if (p->tokens > kMost) {
    set_error("tokens=%d above %d", p->tokens, kMost);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (p->d_ff % p->n_blocks || p->d_model % 64 || p->d_ff / p->n_blocks % 64) {
    set_error("d_model=%d and d_ff / n_blocks=%d / %d must be multiples of 64", p->d_model, p->d_ff, p->n_blocks);
    return UNIF_MOE_ERR_SHAPE;
  }
  const unif_moe_thresholds& th = p->th;
  if (th.topk_fixed < 0 || th.topk_fixed > p->n_experts || isinf(th.tau) || isinf(th.alpha_fixed) ||
      isinf(th.beta_fixed) || (!isnan(th.alpha_fixed) && !(th.alpha_fixed >= 0.f && th.alpha_fixed <= 1.f))) {
    set_error("bad thresholds (topk_fixed=%d, alpha_fixed=%g)", th.topk_fixed, th.alpha_fixed);
    return UNIF_MOE_ERR_ARG;
  }
  return UNIF_MOE_OK;
}

// The parts of the workspace, each at a multiple of 256 bytes.
struct Parts {
  int64_t shr, em, alpha, s, n_pairs, pair, members, h, total;
};
Parts parts_of(const unif_moe_few* p) {
  const int64_t T = p->tokens, G = (int64_t)(p->n_experts + 1) * p->n_blocks;
  Parts r{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  r.shr = take(8 * T);
  r.em = take(8 * T);
  r.alpha = take(4 * T);
  r.s = take(4 * T * p->n_experts);
  r.n_pairs = take(4);
  r.pair = take(2 * G);
  r.members = take(8 * (p->n_blocks + p->n_experts));
  r.h = take(2 * (p->n_experts + 1) * T * p->d_ff);
  r.total = at;
  return r;
}

cudaError_t launch_cluster(void (*kernel)(const Params, const int), int grid, int ctas, size_t smem, cudaStream_t s,
                           const Params& p) {
  const cudaError_t e = allow_smem_once(kernel, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid * ctas);
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
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p, ctas);
}

template <int NT, int TOK>
cudaError_t launch_as(const Params& p, int sms, cudaStream_t s) {
  const int G = (p.K + 1) * p.B;
  const bool routes = p.T <= kTogether;
  void (*up)(const Params) = up_kernel<NT, NT == 1, 0>;
  size_t smem = up_smem(G, p.K, p.C, routes, kUpStages, 0);
  if constexpr (NT > 1) {
    // (five stages instead of four, 24 tokens: 130 us and 129)
    auto hold = [&](int stages, void (*kernel)(const Params)) {
      const size_t need = up_smem(G, p.K, p.C, routes, stages, held_bytes(p.T, p.d));
      if (need > kSmemMost) return false;
      up = kernel;
      smem = need;
      return true;
    };
    if (!hold(4, up_kernel<NT, false, 4>) && !hold(3, up_kernel<NT, false, 3>)) hold(2, up_kernel<NT, false, 2>);
  }
  cudaError_t e;
  if (!routes) {
    const size_t bytes = 4 * (size_t)route_floats(p.C, kWarps);
    e = allow_smem_once(route_kernel, bytes);
    if (e == cudaSuccess) e = launch_dependent(route_kernel, dim3(p.T), dim3(kThreads), bytes, s, p);
    if (e != cudaSuccess) return e;
  }
  e = allow_smem_once(up, smem);
  if (e == cudaSuccess) e = launch_dependent(up, dim3(sms), dim3(32 * kUpWarps), smem, s, p);
  if (e != cudaSuccess) return e;
  // a cluster to 16 output features, of as many CTAs as the SMs hold at once
  const int groups = p.d / 16, slots = 2 * sms;
  int ctas = 8;
  while (ctas > 1 && groups * ctas > slots) ctas /= 2;
  return launch_cluster(down_kernel<NT, TOK>, groups, ctas, down_smem<TOK>(G), s, p);
}

cudaError_t launch(const Params& p, int sms, cudaStream_t s) {
  if (p.T <= 8) return launch_as<1, 8>(p, sms, s);
  if (p.T <= 16) return launch_as<2, 16>(p, sms, s);
  if (p.T <= 32) return launch_as<4, 32>(p, sms, s);
  return launch_as<4, 64>(p, sms, s);
}

bool off(const void* p, uintptr_t by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }

int run(const unif_moe_few* d, const void* x, int64_t ld_x, const void* router, const float* bias, const void* up,
        const void* down, const uint8_t* mask, void* out, int64_t ld_out, int32_t* b_out, int32_t* k_out,
        void* workspace, int64_t workspace_bytes, cudaStream_t s) {
  if (d->tokens == 0) return UNIF_MOE_OK;
  if (!x || !router || !up || !down || !out) {
    set_error("x, router, weights or out is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  if (ld_x < d->d_model || ld_out < d->d_model) {
    set_error("a row stride is below d_model=%d", d->d_model);
    return UNIF_MOE_ERR_ARG;
  }
  if (off(x, 16) || ld_x % 8 || off(router, 16) || off(up, 32) || off(down, 32)) {
    set_error("rows of x and the router must start at multiples of 16 bytes, the weights at one of 32");
    return UNIF_MOE_ERR_ARG;
  }
  const Parts at = parts_of(d);
  if (!workspace || workspace_bytes < at.total) {
    set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)at.total);
    return UNIF_MOE_ERR_CAPACITY;
  }
  if (off(workspace, 16)) {
    set_error("the workspace must be 16-byte aligned");
    return UNIF_MOE_ERR_ARG;
  }
  // (x's rows are read before the first of out's is written)
  const int64_t T = d->tokens, weight_bytes = ((int64_t)d->n_experts + 1) * d->d_ff * d->d_model * 2;
  const Block to{out, ld_out * 2, d->d_model * 2ll, T}, used = flat(workspace, at.total),
      bx{x, ld_x * 2, d->d_model * 2ll, T}, br = flat(router, (1ll + d->n_experts + d->n_blocks) * d->d_model * 2),
      bb = flat(bias, 4ll * (d->n_experts + 1)), bu = flat(up, weight_bytes), bd = flat(down, weight_bytes), bm = flat(mask, T),
      nb = flat(b_out, 4 * T), nk = flat(k_out, 4 * T);
  if (overlap_any(to, {br, bb, bu, bd, bm, nb, nk, used}) || overlap_any(used, {bx, br, bb, bu, bd, bm, nb, nk}) ||
      overlap_any(nb, {bx, br, bb, bu, bd, bm, nk}) || overlap_any(nk, {bx, br, bb, bu, bd, bm})) {
    set_error("out, the counts or the workspace overlaps another array of the call (x under out excepted)");
    return UNIF_MOE_ERR_ARG;
  }
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != UNIF_MOE_OK) return rc;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Params p{};
  p.T = d->tokens; p.d = d->d_model; p.H = d->d_ff; p.K = d->n_experts; p.B = d->n_blocks;
  p.M = p.H / p.B;
  p.C = 1 + p.K + p.B;
  p.tau = isnan(d->th.tau) ? (float)((double)(p.B - 1) / ((double)p.B * p.B)) : d->th.tau;
  p.alpha_fixed = d->th.alpha_fixed;
  p.beta_fixed = d->th.beta_fixed;
  p.topk_fixed = d->th.topk_fixed;
  p.prefix = d->th.prefix_blocks;
  p.x = static_cast<const __nv_bfloat16*>(x);
  p.ld_x = ld_x;
  p.router = static_cast<const __nv_bfloat16*>(router);
  p.bias = bias;
  p.up = static_cast<const __nv_bfloat16*>(up);
  p.down = static_cast<const __nv_bfloat16*>(down);
  p.mask = mask;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.ld_out = ld_out;
  p.b_out = b_out;
  p.k_out = k_out;
  p.shr = reinterpret_cast<uint64_t*>(ws + at.shr);
  p.em = reinterpret_cast<uint64_t*>(ws + at.em);
  p.alpha = reinterpret_cast<float*>(ws + at.alpha);
  p.s = reinterpret_cast<float*>(ws + at.s);
  p.n_pairs = reinterpret_cast<int*>(ws + at.n_pairs);
  p.pair = reinterpret_cast<uint16_t*>(ws + at.pair);
  p.members = reinterpret_cast<uint64_t*>(ws + at.members);
  p.h = reinterpret_cast<__nv_bfloat16*>(ws + at.h);
  const cudaError_t e = launch(p, sms, s);
  if (e != cudaSuccess) {
    set_error("few tokens: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

// The description of a layer's forward of T tokens.
int of_layer(const unif_moe_layer* L, int T, unif_moe_few* d) {
  if (!L) { set_error("NULL handle"); return UNIF_MOE_ERR_ARG; }
  if (L->dtype != UNIF_MOE_BF16) {
    set_error("few tokens: the layer must be bf16");
    return UNIF_MOE_ERR_SHAPE;
  }
  if (!L->loaded) { set_error("forward before load_weights"); return UNIF_MOE_ERR_STATE; }
  *d = unif_moe_few{T, L->d, L->H, L->K, L->B, L->th};
  d->th.tau = L->tau;
  return check(d);
}

}  // namespace few
}  // namespace unif

using unif::set_error;
namespace fw = unif::few;

extern "C" {

int unif_moe_router_table(int d_model, int d_ff, int n_experts, int n_blocks, const void* w_router, const void* w_up,
                          void* table, void* stream) {
  set_error("%s", "");
  const unif_moe_few d{1, d_model, d_ff, n_experts, n_blocks, {NAN, NAN, NAN, 0, 0}};
  const int rc = fw::check(&d);
  if (rc != UNIF_MOE_OK) return rc;
  if (!w_router || !w_up || !table) {
    set_error("w_router, w_up or table is NULL");
    return UNIF_MOE_ERR_ARG;
  }
  const cudaError_t e = unif::launch_dependent(
      fw::table_kernel, dim3((d_model + 255) / 256, 1 + n_experts + n_blocks), dim3(256), 0,
      static_cast<cudaStream_t>(stream), d_model, n_experts, n_blocks, d_ff / n_blocks,
      static_cast<const __nv_bfloat16*>(w_router), static_cast<const __nv_bfloat16*>(w_up),
      static_cast<__nv_bfloat16*>(table));
  if (e != cudaSuccess) {
    set_error("router table: %s", cudaGetErrorString(e));
    return UNIF_MOE_ERR_CUDA;
  }
  return UNIF_MOE_OK;
}

int64_t unif_moe_few_workspace(const unif_moe_few* p) {
  set_error("%s", "");
  return fw::check(p) == UNIF_MOE_OK ? fw::parts_of(p).total : -1;
}

int unif_moe_few_forward(const unif_moe_few* p, const void* x, int64_t ld_x, const void* router, const float* bias,
                         const void* w_up, const void* w_down, const uint8_t* mask, void* out, int64_t ld_out,
                         int32_t* b_out, int32_t* k_out, void* workspace, int64_t workspace_bytes, void* stream) {
  set_error("%s", "");
  const int rc = fw::check(p);
  if (rc != UNIF_MOE_OK) return rc;
  return fw::run(p, x, ld_x, router, bias, w_up, w_down, mask, out, ld_out, b_out, k_out, workspace, workspace_bytes,
                 static_cast<cudaStream_t>(stream));
}

int64_t unif_moe_forward_few_workspace(unif_moe_t L, int T) {
  set_error("%s", "");
  unif_moe_few d;
  return fw::of_layer(L, T, &d) == UNIF_MOE_OK ? fw::parts_of(&d).total : -1;
}

int unif_moe_forward_few(unif_moe_t L, const void* x, int64_t ld_x, int T, const uint8_t* mask, void* out,
                         int64_t ld_out, int32_t* b_out, int32_t* k_out, void* workspace, int64_t workspace_bytes,
                         void* stream) {
  set_error("%s", "");
  unif_moe_few d;
  const int rc = fw::of_layer(L, T, &d);
  if (rc != UNIF_MOE_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || (dev != L->device && cudaSetDevice(L->device) != cudaSuccess)) {
    set_error("no CUDA device");
    return UNIF_MOE_ERR_CUDA;
  }
  const int r = fw::run(&d, x, ld_x, L->wr_bf, L->bias, L->w_up, L->w_down, mask, out, ld_out, b_out, k_out,
                        workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
  if (dev != L->device) cudaSetDevice(dev);
  return r;
}

}  // extern "C"

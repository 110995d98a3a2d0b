// Products in 8-bit integers with a scale for each token and each output channel.
//
//   quantize_rows_kernel  codes[t, i] = round(127 x[t, i] / a_t), scale[t] = a_t / 127, a_t = max |x[t, :]|
//   linear_int_kernel     y[t, n] = (sum_i codes[t, i] W[n, i]) scale[t] w_scale[n] + bias[n], the sum exact in 32-bit integers;
//                         grouped: rows offsets[e] .. offsets[e + 1] go through weight set e
//   combine_kernel        out[t, :] = sum_j weight[t, j] y[position[t, j], :]
//   combine_grad_kernel   d_weight[t, j] = <d_out[t, :], y[position[t, j], :]>,  d_y[position[t, j], :] = weight[t, j] d_out[t, :]
#include "op_common.cuh"
#include "tc_common.cuh"

using namespace mix;
using namespace mix::tc;

namespace {

// ---------------------------------------------------------------------------------------------------- quantisation
// A row's codes are the exact quotients 127 x / a rounded to the nearest, halves to the even one.  A division costs more than the
// rest of the row's work, so the quotient comes from a multiplication by 127 / a, and adding 1.5 * 2^23 (in the same instruction)
// rounds to a whole number, whose two's complement is in the low bits of the sum.  That is exact:
//   x = X 2^f and a = A 2^e with whole X, A < 2^11 (fp16; 2^8 for bf16).  A quotient that is no half differs from the nearest half
//   (2n + 1) / 2 by |254 X 2^f - (2n + 1) A 2^e| / (2 A 2^e), at least 2^(f - e) / 2^12, which relative to the quotient is 9.6e-7 or
//   more; the factor, nudged up by one step, is off by 1.8e-7 at most.
//   A half needs 127 | (2n + 1) A.  If 127 does not divide A that is 2n + 1 = 127 alone: x = a / 2, 63.5, and the factor nudged up
//   takes it to 64, the even one.  If A = 127 2^j the factor is a power of two and everything is exact.  Other multiples of 127 (eight
//   largest values of fp16 in 1024) go by division; so do rows that lie so far from 1 that 127 x or 127 / a would leave fp32's
//   range, scaled by a power of two first.
// 8192 rows of 8192 bf16: 60 us with a rounding, a comparison and a conversion per element, 51 with a test for halves, 36.6 so (5.5 TB/s).
template <typename T>
struct Pair2;
template <>
struct Pair2<__nv_bfloat16> {
  using V = __nv_bfloat162;
  static __device__ __forceinline__ float2 f32(V v) { return __bfloat1622float2(v); }
};
template <>
struct Pair2<__half> {
  using V = __half2;
  static __device__ __forceinline__ float2 f32(V v) { return __half22float2(v); }
};
// Largest size of 8 elements; NaN where one is NaN.
template <typename T>
__device__ __forceinline__ typename Pair2<T>::V sizes8(const uint4& raw, typename Pair2<T>::V a) {
  const typename Pair2<T>::V* e = reinterpret_cast<const typename Pair2<T>::V*>(&raw);
#pragma unroll
  for (int j = 0; j < 4; ++j) a = __hmax2_nan(a, __habs2(e[j]));
  return a;
}
template <typename T>
__device__ __forceinline__ uint2 codes8(const uint4& raw, float factor) {
  const typename Pair2<T>::V* e = reinterpret_cast<const typename Pair2<T>::V*>(&raw);
  unsigned t[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = Pair2<T>::f32(e[j]);
    t[2 * j] = __float_as_uint(fmaf(f.x, factor, 12582912.f));
    t[2 * j + 1] = __float_as_uint(fmaf(f.y, factor, 12582912.f));
  }
  uint2 c;
  c.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
  c.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
  return c;
}
template <typename T>
__device__ __noinline__ uint2 codes8_divided(const uint4& raw, float a) {
  const float pre = a > 1e30f ? 0x1p-64f : (a < 1e-30f ? 0x1p64f : 1.f);
  const T* e = reinterpret_cast<const T*>(&raw);
  uint2 c;
  signed char* b = reinterpret_cast<signed char*>(&c);
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = (signed char)(int)rintf(__fdiv_rn(127.f * (to_f32(e[j]) * pre), a * pre));
  return c;
}

constexpr int kQuantVecs = 4;                                  // 8-element vectors a thread keeps
template <typename T, int THREADS, bool vec>
__global__ void __launch_bounds__(THREADS < 128 ? 128 : THREADS, THREADS == 256 ? 6 : (THREADS == 128 ? 12 : 9))
quantize_rows_kernel(const T* __restrict__ x, long long ld, int x_rows, const int* __restrict__ order, int div, int n_rows, int d,
                     signed char* __restrict__ codes, float* __restrict__ scale) {
  constexpr int kRows = THREADS < 128 ? 128 / THREADS : 1;     // rows a CTA takes
  __shared__ unsigned red[kRows == 1 ? THREADS / 32 : 1];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x % THREADS;
  const long long i = (long long)blockIdx.x * kRows + threadIdx.x / THREADS;
  if (i >= n_rows) return;                                     // (whole warps; a CTA of one row has it)
  long long src = i;
  if (order) {
    const int o = order[i];
    src = o < 0 ? -1 : o / div;
    if (src >= x_rows) src = -1;
  }
  const int n_vec = d / 8;                                     // (d is a multiple of 16)
  uint2* out = reinterpret_cast<uint2*>(codes + i * d);
  if (src < 0) {                                               // an entry without a token: zeros
    for (int v = tid; v < n_vec; v += THREADS) out[v] = make_uint2(0u, 0u);
    if (tid == 0) scale[i] = 0.f;
    return;
  }
  const T* row = x + src * ld;
  using V = typename Pair2<T>::V;
  uint4 keep[kQuantVecs];
  V most;
  most.x = most.y = from_f32<T>(0.f);
  auto fetch = [&](int v) -> uint4 {
    if (vec) return *reinterpret_cast<const uint4*>(row + 8ll * v);
    uint4 raw;
    T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = row[8ll * v + j];
    return raw;
  };
#pragma unroll
  for (int b = 0; b < kQuantVecs; ++b) {
    const int v = tid + b * THREADS;
    keep[b] = v < n_vec ? fetch(v) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int b = 0; b < kQuantVecs; ++b) most = sizes8<T>(keep[b], most);
  for (int v = tid + kQuantVecs * THREADS; v < n_vec; v += THREADS) most = sizes8<T>(fetch(v), most);
  const float2 two = Pair2<T>::f32(most);
  // (sizes compare as their bits do, and a NaN's are above infinity's)
  unsigned bits = __reduce_max_sync(0xffffffffu, max(__float_as_uint(two.x) & 0x7fffffffu, __float_as_uint(two.y) & 0x7fffffffu));
  if (kRows == 1 && THREADS > 32) {
    if ((tid & 31) == 0) red[tid >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) bits = max(bits, red[w]);
  }
  const float a = __uint_as_float(bits);
  if (!(a < INFINITY)) {                                       // a row with an infinity or a NaN: its products are NaN
    for (int v = tid; v < n_vec; v += THREADS) out[v] = make_uint2(0u, 0u);
    if (tid == 0) scale[i] = __int_as_float(0x7fc00000);
    return;
  }
  const unsigned digits = (bits & 0x7fffffu) | 0x800000u, by127 = digits / 127u;
  const bool multiple = by127 * 127u == digits, exact = multiple && (by127 & (by127 - 1u)) == 0u;
  if (a == 0.f) {
    for (int v = tid; v < n_vec; v += THREADS) out[v] = make_uint2(0u, 0u);
  } else if (a >= 1e-30f && a <= 1e30f && (!multiple || exact)) {
    const float factor = __uint_as_float(__float_as_uint(__fdiv_rn(127.f, a)) + (exact ? 0u : 1u));
#pragma unroll
    for (int b = 0; b < kQuantVecs; ++b) {
      const int v = tid + b * THREADS;
      if (v < n_vec) out[v] = codes8<T>(keep[b], factor);
    }
    for (int v = tid + kQuantVecs * THREADS; v < n_vec; v += THREADS) out[v] = codes8<T>(fetch(v), factor);
  } else {
    for (int v = tid; v < n_vec; v += THREADS) out[v] = codes8_divided<T>(fetch(v), a);
  }
  if (tid == 0) scale[i] = __fdiv_rn(a, 127.f);
}

// ---------------------------------------------------------------------------------------------------- the product
// A tile is 128 output channels x NT tokens: the WEIGHTS are the matrix operand with 128 rows and the tokens the one with NT, so
// that a few tokens (a decode step, an expert's share) make a narrow tile and not one of mostly empty rows.  Accumulators are
// 32-bit integers in tensor memory, two of them, so that one tile is written out while the next is computed.
constexpr int kTileCh = 128;                                   // output channels of a tile
constexpr int kKBytes = 128;                                   // codes of a row in a stage: one swizzled 128-byte line
constexpr int kEpiWarps = 8;                                   // two for each quarter of tensor memory's lanes
constexpr int kGemmThreads = 64 + 32 * kEpiWarps;              // copies, tensor-core instructions, epilogue
constexpr int kStageOut = 2048;                                // bytes of a warp's piece of the output on its way to memory
constexpr long long kI8WaitCycles = 4000000000ll;              // about two seconds
constexpr long long kI8WaitCyclesTest = 2000000ll;             // ~1 ms: the cap under mix_debug_linear_int_stall

__device__ unsigned g_i8_status;                               // MIX_STATUS_WAIT_TIMEOUT, until mix_linear_int_status reads it
std::atomic<int> g_i8_test_stall;                              // host: calls are launched with the test's stall

// kPair: two CTAs of a cluster work on one tile of 256 channels with cta_group::2.  Each holds its own 128 channels and half of the
// tokens' rows, so that a k-block of 256 tokens costs a CTA 32 KB of copies and 32 KB of reads of shared memory, not 48 and 48:
// at 128 bytes a clock the single CTA's 96 KB take 768 clocks, while the tensor core needs 512 (measured 834 and 1573 us for
// 8192 x 8192 x 32768).
//
// kSplit: the 2, 4 or 8 CTAs of a cluster work on one tile, each on its part of the codes of a row, for calls whose tiles leave most
// SMs without one (4096 channels are 32).  The parts meet in shared memory, in 32-bit integers: where they are added up does not
// show in the result.
enum { kSingle = 0, kPairs = 1, kSplit = 2 };
constexpr int kMostParts = 8;
template <int NT, int kMode>
struct GemmCfg {
  static constexpr bool kPair = kMode == kPairs;
  static constexpr int kCtas = kPair ? 2 : 1;
  static constexpr int kTokRows = NT / kCtas;                  // rows of the token operand in this CTA's shared memory
  static constexpr int kBoxRows = kTokRows < 64 ? kTokRows : 64;   // tokens of a copy
  static constexpr int kABytes = kTileCh * kKBytes;
  static constexpr int kStageBytes = kABytes + kTokRows * kKBytes;
  static constexpr int kStages = (200 * 1024) / kStageBytes < 12 ? (200 * 1024) / kStageBytes : 12;
  static constexpr int kTmemCols = 2 * NT < 32 ? 32 : 2 * NT;
  static constexpr int kSmem = kStages * kStageBytes + kEpiWarps * kStageOut + 1024;
  static_assert(NT * kTileCh * 4 <= kStages * kStageBytes, "a part's sums fit where its operands were");
};

struct GemmShared {
  unsigned long long full[12], empty[12], acc_full[2], acc_empty[2];
  unsigned tmem_base;
  int abort_flag;
  long long wait_cycles;                                       // cap of every bounded wait in this launch
  int row0[kOpMaxExperts + 1];                                 // rows of expert e: row0[e] .. row0[e + 1]
  int tile0[kOpMaxExperts + 1];                                // tiles of expert e
};

// kind::i8: 32-bit integer accumulators, both operands signed, both K-major; K = 32 codes an instruction
__host__ __device__ constexpr unsigned idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)(n >> 3) << 17) | ((unsigned)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate,
                                        unsigned on) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}

__device__ __forceinline__ void umma_i8_pair(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate,
                                             unsigned on) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}

struct I8Tile {
  int expert, ch0, row0, n_tok;
  bool once;                                                   // no other tile reads these channels of W
};

// Tiles of an expert: groups of kGroup token tiles; in a group the channels one after the other, each with all of the group's
// token tiles next to each other: a tile of W comes from DRAM once a group, and the group's tokens stay in L2.  (8192 x 8192 codes by
// 32768 channels with their quantisation, back to back under the power cap: 1495 us; groups of 8 1513, of 4 or 32 1607.)
constexpr int kGroup = 16;
__device__ __forceinline__ void i8_place(int local, int tt, int ch_tiles, int* ch, int* tk) {
  const int group = local / (kGroup * ch_tiles), in = local - group * kGroup * ch_tiles, wide = min(kGroup, tt - group * kGroup);
  *ch = in / wide;
  *tk = group * kGroup + in % wide;
}
// The tiles of the last wave, where they leave half of the workers or more without one, are cut into `pieces` along the tokens: a piece
// of a tile of 250 tokens takes a little more than half its time, and 1000 x 5120 codes by 9992 channels -- 160 tiles for 74 pairs --
// 39.9 us instead of 41.5.  In pairs only: other tiles are narrow as they are.
struct LastWave {
  int first, pieces;                                           // numbers from `first` on are pieces
};
__device__ __forceinline__ LastWave last_wave(int tiles, int n_workers, int tile_tok) {
  const int left = tiles % n_workers;
  LastWave w = {tiles - left, left == 0 ? 1 : min(min(n_workers / left, tile_tok / 32), 8)};
  return w;
}
template <bool kPair>
__device__ __forceinline__ I8Tile i8_tile(const GemmShared* sh, int tile, int ch_tiles, int tile_tok, const LastWave& last, int& e) {
  int piece = 0, pieces = 1;
  if (kPair && tile >= last.first) {
    const int x = tile - last.first;
    pieces = last.pieces;
    piece = x % pieces;
    tile = last.first + x / pieces;
  }
  while (tile >= sh->tile0[e + 1]) ++e;                        // (a role's tiles only rise)
  const int rows = sh->row0[e + 1] - sh->row0[e], tt = (rows + tile_tok - 1) / tile_tok;
  int ch, tk;
  i8_place(tile - sh->tile0[e], tt, ch_tiles, &ch, &tk);
  I8Tile t;
  t.expert = e;
  t.once = tt == 1 && pieces == 1;
  t.ch0 = ch * (kPair ? 2 * kTileCh : kTileCh);
  // an expert's rows are dealt evenly: with a full tile and a small one in turn, the even workers would get all the full ones
  const int each = ((rows + tt - 1) / tt + 15) & ~15;
  t.row0 = sh->row0[e] + tk * each;
  t.n_tok = min(each, rows - tk * each);                       // (0 or less: the tiles in front of this one hold all rows)
  if (pieces > 1) {
    const int part = ((t.n_tok + pieces - 1) / pieces + 31) & ~31;
    t.row0 += piece * part;
    t.n_tok = min(part, t.n_tok - piece * part);
  }
  return t;
}

template <typename OutT, int NT, int kMode>
__global__ void __launch_bounds__(kGemmThreads, 1)
linear_int_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const float* __restrict__ scale,
                  const float* __restrict__ w_scale, const float* __restrict__ bias, const int* __restrict__ offsets, int n_rows, int K,
                  int N, int E, int tile_tok, int parts, OutT* __restrict__ out, long long ld_out, int vec, int test_stall) {
  using Cfg = GemmCfg<NT, kMode>;
  constexpr bool kPair = Cfg::kPair;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  __shared__ GemmShared shared;
  __shared__ float tok_scale[kEpiWarps][NT];                   // a copy per warp of the epilogue
  GemmShared* sh = &shared;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = kPair ? (int)cluster_ctarank() : 0;         // rank 0 leads a pair: it issues the instructions, and its barriers count both CTAs' copies
  const int part = kMode == kSplit ? (int)cluster_ctarank() : 0;
  const int share = kPair ? 2 : (kMode == kSplit ? parts : 1);
  const int worker = (int)blockIdx.x / share, n_workers = (int)gridDim.x / share;
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&sh->acc_full[a]), 1);
      mbar_init(smem_u32(&sh->acc_empty[a]), kEpiWarps * Cfg::kCtas);
    }
    sh->abort_flag = 0;
    sh->wait_cycles = test_stall ? kI8WaitCyclesTest : kI8WaitCycles;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (kPair) tmem_alloc_pair(smem_u32(&sh->tmem_base), Cfg::kTmemCols);
    else tmem_alloc(smem_u32(&sh->tmem_base), Cfg::kTmemCols);
  }
  constexpr int kChannels = kTileCh * Cfg::kCtas;
  const int ch_tiles = (N + kChannels - 1) / kChannels;
  const int num_kb = (K + kKBytes - 1) / kKBytes;
  const int kb0 = kMode == kSplit ? num_kb * part / parts : 0, kb1 = kMode == kSplit ? num_kb * (part + 1) / parts : num_kb;
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) {                                             // the experts' rows and tiles; offsets that fall or leave the rows are held in
    int row = 0, tiles = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + lane;
      int end = offsets ? (e < E ? min(max(offsets[e + 1], 0), n_rows) : 0) : n_rows;
      const int begin = offsets ? (e < E ? min(max(offsets[e], 0), n_rows) : 0) : 0;
      if (e0 == 0) row = __shfl_sync(0xffffffffu, begin, 0);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {                       // running maximum: never below an earlier offset
        const int y = __shfl_up_sync(0xffffffffu, end, o);
        if (lane >= o) end = max(end, y);
      }
      end = max(end, row);
      int prev = __shfl_up_sync(0xffffffffu, end, 1);
      if (lane == 0) prev = row;
      int n = e < E ? (end - prev + tile_tok - 1) / tile_tok * ch_tiles : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, n, o);
        if (lane >= o) n += y;
      }
      if (e < E) {
        sh->row0[e + 1] = end;
        sh->tile0[e + 1] = tiles + n;
        if (e == 0) {
          sh->row0[0] = prev;
          sh->tile0[0] = 0;
        }
      }
      row = __shfl_sync(0xffffffffu, end, 31);
      tiles += __shfl_sync(0xffffffffu, n, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (kPair) cluster_sync_all();                               // the peer's barriers are initialised before anything is sent to them
  tc_fence_after();
  const unsigned tmem_base = (unsigned)uniform((int)sh->tmem_base);
  const int tiles = uniform(sh->tile0[E]);
  const LastWave last = !kPair ? LastWave{tiles, 1} : last_wave(tiles, n_workers, tile_tok);
  const int total = kPair ? last.first + (tiles - last.first) * last.pieces : tiles;
  const long long* cap = &sh->wait_cycles;

  if (warp == 0) {
    int stage = 0, e = 0;
    unsigned phase = 0;
    bool ok = true;
    const unsigned long long stream = l2_evict_first();
    for (int tile = worker; tile < total && ok; tile += n_workers) {
      const I8Tile t = i8_tile<kPair>(sh, tile, ch_tiles, tile_tok, last, e);
      if (t.n_tok <= 0) continue;
      const int tok_rows = kPair ? ((t.n_tok + 31) & ~31) / 2 : t.n_tok;     // of this CTA
      const int boxes = uniform((tok_rows + Cfg::kBoxRows - 1) / Cfg::kBoxRows);
      // (E * N rows of W fit in 31 bits: checked on the host.  Channels behind the last and tokens behind the expert's are
      // other rows or the fill value; what comes of them is not stored)
      const int wy = uniform(t.expert * N + t.ch0 + rank * kTileCh), xy = uniform(t.row0 + (kPair ? rank * tok_rows : 0));
      const bool once = uniform((int)t.once) != 0;             // (then what the kernels around this one share stays in L2)
      const unsigned bytes = (Cfg::kABytes + boxes * Cfg::kBoxRows * kKBytes) * Cfg::kCtas;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_bounded_warp(smem_u32(&sh->empty[stage]), phase ^ 1u, &sh->abort_flag, cap, &g_i8_status)) { ok = false; break; }
        if (test_stall) { ok = false; break; }                 // no stage is ever filled: the waits of the others run out
        const unsigned bar = smem_u32(&sh->full[stage]), sa = smem_u32(ring + stage * Cfg::kStageBytes), on = elect_one();
        if (kPair) {
          if (rank == 0) mbar_expect_tx(bar, bytes, on);
          const unsigned bar_c = mapa_cluster(bar, 0);
          if (once) tma_load_2d_pair_hint(sa, &tmap_w, kb * kKBytes, wy, bar_c, stream, on);
          else tma_load_2d_pair(sa, &tmap_w, kb * kKBytes, wy, bar_c, on);
          for (int b = 0; b < boxes; ++b)
            tma_load_2d_pair(sa + Cfg::kABytes + b * Cfg::kBoxRows * kKBytes, &tmap_x, kb * kKBytes, xy + b * Cfg::kBoxRows, bar_c, on);
        } else {
          mbar_expect_tx(bar, bytes, on);
          if (once) tma_load_2d_hint(sa, &tmap_w, kb * kKBytes, wy, bar, stream, on);
          else tma_load_2d(sa, &tmap_w, kb * kKBytes, wy, bar, on);
          for (int b = 0; b < boxes; ++b)
            tma_load_2d(sa + Cfg::kABytes + b * Cfg::kBoxRows * kKBytes, &tmap_x, kb * kKBytes, xy + b * Cfg::kBoxRows, bar, on);
        }
        if (++stage == Cfg::kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      int stage = 0, e = 0;
      unsigned phase = 0, acc = 0, acc_phase = 0;
      bool ok = true;
      for (int tile = worker; tile < total && ok; tile += n_workers) {
        const I8Tile t = i8_tile<kPair>(sh, tile, ch_tiles, tile_tok, last, e);
        if (t.n_tok <= 0) continue;
        const unsigned idesc = (unsigned)uniform((int)(kPair ? idesc_i8(2 * kTileCh, (t.n_tok + 31) & ~31) : idesc_i8(kTileCh, (t.n_tok + 15) & ~15)));
        if (!mbar_wait_bounded_warp(smem_u32(&sh->acc_empty[acc]), acc_phase ^ 1u, &sh->abort_flag, cap, &g_i8_status)) break;
        tc_fence_after();
        const unsigned d_tmem = tmem_base + acc * NT;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait_bounded_warp(smem_u32(&sh->full[stage]), phase, &sh->abort_flag, cap, &g_i8_status)) { ok = false; break; }
          tc_fence_after();
          const unsigned sa = smem_u32(ring + stage * Cfg::kStageBytes);
          const unsigned long long da = umma_desc(sa), db = umma_desc(sa + Cfg::kABytes);
          const unsigned on = elect_one();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (kPair) umma_i8_pair(d_tmem, da + 2ull * k, db + 2ull * k, idesc, (unsigned)((kb - kb0) | k) != 0u, on);
            else umma_i8(d_tmem, da + 2ull * k, db + 2ull * k, idesc, (unsigned)((kb - kb0) | k) != 0u, on);
          }
          if (kPair) umma_commit_pair(smem_u32(&sh->empty[stage]), on);      // the stage is free again, in both CTAs
          else umma_commit(smem_u32(&sh->empty[stage]), on);
          if (++stage == Cfg::kStages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (kPair) umma_commit_pair(smem_u32(&sh->acc_full[acc]), elect_one());
        else umma_commit(smem_u32(&sh->acc_full[acc]), elect_one());
        acc ^= 1u;
        if (acc == 0) acc_phase ^= 1u;
      }
    }
  } else {
    // Epilogue.  A thread has one channel and 32 tokens of it, the output wants channels next to each other: the warp's 32 x 32
    // piece goes through shared memory and leaves in 16-byte vectors, 64 bytes a token (128 for fp32).  Storing element by element
    // from the registers costs 12 instructions an element, with four warps more time than the products of 2048 codes.
    const int q = warp & 3;                                    // tensor-memory lanes this warp may read
    const int half = (warp - 2) >> 2;                          // every other piece of 32 tokens
    constexpr int kTok = kStageOut / (32 * (int)sizeof(OutT)); // tokens of a piece: 32, or 16 of fp32
    constexpr int kVW = 16 / (int)sizeof(OutT), kLanesRow = 32 / kVW, kRowsStep = 32 / kLanesRow;
    int e = 0;
    unsigned acc = 0, acc_phase = 0;
    float* my_scale = tok_scale[warp - 2];
    OutT* piece = reinterpret_cast<OutT*>(ring + Cfg::kStages * Cfg::kStageBytes + (warp - 2) * kStageOut);
    for (int tile = worker; tile < total; tile += n_workers) {
      const I8Tile t = i8_tile<kPair>(sh, tile, ch_tiles, tile_tok, last, e);
      if (t.n_tok <= 0) continue;
      const int ch0 = t.ch0 + rank * kTileCh + q * 32, ch = ch0 + lane;
      const bool valid = ch < N;
      const float ws = valid ? w_scale[(long long)t.expert * N + ch] : 0.f;
      const float bs = valid && bias ? bias[(long long)t.expert * N + ch] : 0.f;
      __syncwarp();
      for (int i = lane; i < t.n_tok; i += 32) my_scale[i] = scale[t.row0 + i];
      __syncwarp();
      if (!mbar_wait_bounded_warp(smem_u32(&sh->acc_full[acc]), acc_phase, &sh->abort_flag, cap, &g_i8_status)) break;
      tc_fence_after();
      const unsigned taddr = tmem_base + acc * NT + ((unsigned)(q * 32) << 16);
      if (kMode == kSplit) {                                   // the part's sums, [token][channel], where the operands were (all of them are used up)
        int* sums = reinterpret_cast<int*>(ring) + q * 32 + lane;
        for (int c0 = half * 32; c0 < t.n_tok; c0 += 64) {
          float v[32];
          tmem_ld32(taddr + c0, v);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (c0 + i < t.n_tok) sums[(c0 + i) * kTileCh] = __float_as_int(v[i]);
        }
        continue;                                              // (a call has a tile per cluster at most)
      }
      for (int c0 = half * 32; c0 < t.n_tok; c0 += 64) {
        float v[32];
        tmem_ld32(taddr + c0, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = fmaf((float)__float_as_int(v[i]) * my_scale[c0 + i], ws, bs);
#pragma unroll
        for (int p = 0; p < 32; p += kTok) {
#pragma unroll
          for (int i = 0; i < kTok; ++i) piece[i * 32 + lane] = from_f32<OutT>(v[p + i]);
          __syncwarp();
          OutT* dst = out + (long long)(t.row0 + c0 + p) * ld_out + ch0;
          const int n = min(kTok, t.n_tok - c0 - p);
          if (vec) {
            const int col = lane % kLanesRow * kVW;
#pragma unroll
            for (int i = 0; i < kTok; i += kRowsStep) {
              const int r = i + lane / kLanesRow;
              if (r < n && ch0 + col < N) {
                if (ch0 + col + kVW <= N) {
                  *reinterpret_cast<uint4*>(dst + r * ld_out + col) = *reinterpret_cast<const uint4*>(piece + r * 32 + col);
                } else {
                  for (int j = 0; ch0 + col + j < N; ++j) dst[r * ld_out + col + j] = piece[r * 32 + col + j];
                }
              }
            }
          } else if (valid) {
            for (int r = 0; r < n; ++r) dst[r * ld_out + lane] = piece[r * 32 + lane];
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (kPair) mbar_arrive_cluster(mapa_cluster(smem_u32(&sh->acc_empty[acc]), 0));
        else mbar_arrive(smem_u32(&sh->acc_empty[acc]));
      }
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (sh->abort_flag) {                                        // copies in flight land before shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) __nanosleep(1000);
  }
  if (kMode == kSplit) {
    cluster_sync_all();
    if (worker < total) {                                      // (the same in all CTAs of the cluster) every part writes its share of the tokens
      int e = 0;
      const I8Tile t = i8_tile<kPair>(sh, worker, ch_tiles, tile_tok, last, e);
      const unsigned sums = smem_u32(ring);
      for (int i = threadIdx.x; i < (t.n_tok - part + parts - 1) / parts * (kTileCh / 4); i += kGemmThreads) {   // four channels of a token
        const int row = part + i / (kTileCh / 4) * parts, c = i % (kTileCh / 4) * 4, ch = t.ch0 + c;
        if (ch >= N) continue;
        int4 sum[kMostParts];
#pragma unroll
        for (int r = 0; r < kMostParts; ++r) {
          sum[r] = make_int4(0, 0, 0, 0);
          if (r < parts)
            asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(sum[r].x), "=r"(sum[r].y), "=r"(sum[r].z), "=r"(sum[r].w)
                         : "r"(mapa_cluster(sums + (row * kTileCh + c) * 4, r)));
        }
        int all[4] = {0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < kMostParts; ++r) {
          all[0] += sum[r].x;
          all[1] += sum[r].y;
          all[2] += sum[r].z;
          all[3] += sum[r].w;
        }
        const float by = scale[t.row0 + row];
        const long long w = (long long)t.expert * N + ch;
        __align__(16) OutT v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = ch + j < N ? from_f32<OutT>(fmaf((float)all[j] * by, w_scale[w + j], bias ? bias[w + j] : 0.f)) : from_f32<OutT>(0.f);
        OutT* dst = out + (long long)(t.row0 + row) * ld_out + ch;
        if (vec && ch + 4 <= N) {
          if (sizeof(OutT) == 4) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(v);
          else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(v);
        } else {
          for (int j = 0; j < 4 && ch + j < N; ++j) dst[j] = v[j];
        }
      }
    }
    cluster_sync_all();                                        // the sums stay until they have been read
  }
  if (kPair) cluster_sync_all();                               // neither CTA's barriers or tensor memory go while the other may still reach them
  if (warp == 1) {
    tc_fence_after();
    if (kPair) tmem_dealloc_pair(tmem_base, Cfg::kTmemCols);
    else tmem_dealloc(tmem_base, Cfg::kTmemCols);
  }
}

// ---------------------------------------------------------------------------------------------------- the sum over experts
// A thread has one vector of one token; all of the token's rows are on their way at once.  2048 tokens, 6 of 5120 bf16: 24.2 us
// (6.1 TB/s), 38 with the rows in fours and three vectors a thread.
// The rows are read in the type that the products left them in, which is the caller's choice: 16-bit results are rounded once more than the sum
// needs.  1999 tokens on 6 of 64 experts of 2048 x 5120: the relative error of the bf16 output is 0.0023 with bf16 results between, 0.0017 (its
// own rounding) with fp32 ones, for which the product takes 166 us instead of 155 and the sum, whose output has y's type, 44.5 instead
// of 23.6.
constexpr int kCombineThreads = 128;
template <typename T, int KMAX, bool vec>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const T* __restrict__ y, long long ld_y, int y_rows, const float* __restrict__ weights, const int* __restrict__ position,
               int k, int N, T* __restrict__ out, long long ld_out) {
  constexpr int VW = vec ? RowVec<T>::VW : 1;
  pdl_wait();
  pdl_launch_dependents();
  const long long t = blockIdx.x;
  const int c0 = (blockIdx.y * kCombineThreads + threadIdx.x) * VW;
  if (c0 >= N) return;
  int at[KMAX];
  float w[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    at[j] = j < k ? position[t * k + j] : -1;
    w[j] = j < k ? weights[t * k + j] : 0.f;
  }
  float acc[VW];
#pragma unroll
  for (int i = 0; i < VW; ++i) acc[i] = 0.f;
  if (vec && c0 + VW <= N) {
    uint4 raw[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j)
      if ((unsigned)at[j] < (unsigned)y_rows) raw[j] = *reinterpret_cast<const uint4*>(y + at[j] * ld_y + c0);
#pragma unroll
    for (int j = 0; j < KMAX; ++j)
      if ((unsigned)at[j] < (unsigned)y_rows) {
        const T* e = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
        for (int i = 0; i < VW; ++i) acc[i] = fmaf(w[j], to_f32(e[i]), acc[i]);
      }
    uint4 sum;
    T* e = reinterpret_cast<T*>(&sum);
#pragma unroll
    for (int i = 0; i < VW; ++i) e[i] = from_f32<T>(acc[i]);
    *reinterpret_cast<uint4*>(out + t * ld_out + c0) = sum;
  } else {
    for (int i = 0; i < VW && c0 + i < N; ++i) {
      float a = 0.f;
#pragma unroll
      for (int j = 0; j < KMAX; ++j)
        if ((unsigned)at[j] < (unsigned)y_rows) a = fmaf(w[j], to_f32(y[at[j] * ld_y + c0 + i]), a);
      out[t * ld_out + c0 + i] = from_f32<T>(a);
    }
  }
}

// The gradients.  A CTA has a token: its d_out is read once for all of the token's rows, and the products are added up in a fixed order
// (a thread's vectors, the lanes of a warp, the warps).  8192 tokens, 2 of 4096 bf16: 36.7 us (5.5 TB/s; 49 with the rows one after the
// other), 55 with d_y; 2048 tokens, 6 of 5120: 39 (3.8 TB/s) and 57 -- its 640 vectors are two and a half trips of 256 threads, and
// six rows carry the registers of eight.
constexpr int kCombineGradThreads = 256;
template <typename T, int KMAX, bool vec>
__global__ void __launch_bounds__(kCombineGradThreads)
combine_grad_kernel(const T* __restrict__ y, long long ld_y, int y_rows, const float* __restrict__ weights, const int* __restrict__ position,
                    int k, int N, const T* __restrict__ d_out, long long ld_d, float* __restrict__ d_weights, T* __restrict__ d_y,
                    long long ld_dy) {
  constexpr int VW = vec ? RowVec<T>::VW : 1;
  __shared__ float part[kCombineGradThreads / 32][KMAX];
  pdl_wait();
  pdl_launch_dependents();
  const long long t = blockIdx.x;
  int at[KMAX];
  float w[KMAX], dot[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    at[j] = j < k ? position[t * k + j] : -1;
    w[j] = j < k && d_y ? weights[t * k + j] : 0.f;
    dot[j] = 0.f;
  }
  for (long long c = (long long)threadIdx.x * VW; c < N; c += kCombineGradThreads * VW) {
    const bool whole = vec && c + VW <= N;
    if (whole) {                                               // all rows of the token under way at once
      uint4 raw[KMAX];
      const uint4 graw = *reinterpret_cast<const uint4*>(d_out + t * ld_d + c);
#pragma unroll
      for (int j = 0; j < KMAX; ++j)
        if ((unsigned)at[j] < (unsigned)y_rows) raw[j] = *reinterpret_cast<const uint4*>(y + at[j] * ld_y + c);
      const T* g = reinterpret_cast<const T*>(&graw);
#pragma unroll
      for (int j = 0; j < KMAX; ++j)
        if ((unsigned)at[j] < (unsigned)y_rows) {
          const T* e = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
          for (int i = 0; i < VW; ++i) dot[j] = fmaf(to_f32(g[i]), to_f32(e[i]), dot[j]);
          if (d_y) {
            uint4 out;
            T* d = reinterpret_cast<T*>(&out);
#pragma unroll
            for (int i = 0; i < VW; ++i) d[i] = from_f32<T>(w[j] * to_f32(g[i]));
            *reinterpret_cast<uint4*>(d_y + at[j] * ld_dy + c) = out;
          }
        }
    } else {
      for (int i = 0; i < VW && c + i < N; ++i) {
        const float g = to_f32(d_out[t * ld_d + c + i]);
#pragma unroll
        for (int j = 0; j < KMAX; ++j)
          if ((unsigned)at[j] < (unsigned)y_rows) {
            dot[j] = fmaf(g, to_f32(y[at[j] * ld_y + c + i]), dot[j]);
            if (d_y) d_y[at[j] * ld_dy + c + i] = from_f32<T>(w[j] * g);
          }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    const float s = group_sum<32>(dot[j]);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5][j] = s;
  }
  __syncthreads();
  if (threadIdx.x < k) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kCombineGradThreads / 32; ++i) s += part[i][threadIdx.x];
    d_weights[t * k + threadIdx.x] = s;
  }
}

// ---------------------------------------------------------------------------------------------------- host side
struct Gemm {
  const void* codes;
  const float* scale;
  const void* w;
  const float* w_scale;
  const float* bias;
  const int* offsets;
  int n_rows, K, N, E;
  void* out;
  long long ld_out;
};

long long div_up(long long a, long long b) { return (a + b - 1) / b; }
// Tiles of a call, at most, however the rows fall on the experts.
long long tiles_at_most(const Gemm& g, int tile_tok, int channels) {
  const long long tok = g.E == 1 ? div_up(g.n_rows, tile_tok) : (long long)g.n_rows / tile_tok + (g.E < g.n_rows ? g.E : g.n_rows);
  return tok * div_up(g.N, channels);
}

// Tokens of a tile, and the parts of its codes.
struct TilePlan {
  int mode, nt, tile_tok, parts;
};

template <typename OutT, int NT, int kMode>
cudaError_t gemm_launch(const Gemm& g, const TilePlan& p, int dev, int n_sms, cudaStream_t s) {
  using Cfg = GemmCfg<NT, kMode>;
  static std::atomic<int> ready[kOpDevices];
  if (!ready[dev].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(linear_int_kernel<OutT, NT, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
    if (e != cudaSuccess) return e;
    ready[dev].store(1, std::memory_order_relaxed);
  }
  CUtensorMap tw, tx;
  if (make_tmap_i8(&tw, g.w, (unsigned long long)g.E * g.N, g.K, kTileCh) != MIX_OK || make_tmap_i8(&tx, g.codes, g.n_rows, g.K, Cfg::kBoxRows) != MIX_OK)
    return cudaErrorInvalidValue;
  const int ctas = kMode == kSplit ? p.parts : Cfg::kCtas;
  const long long most = tiles_at_most(g, p.tile_tok, kTileCh * Cfg::kCtas), workers = n_sms / ctas;
  const int vec = (((uintptr_t)g.out | (uintptr_t)(g.ld_out * (long long)sizeof(OutT))) & 15u) == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((most < workers ? most : workers) * ctas));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  int n_at = 0;
  if (ctas > 1) {
    at[n_at].id = cudaLaunchAttributeClusterDimension;
    at[n_at].val.clusterDim.x = ctas;
    at[n_at].val.clusterDim.y = 1;
    at[n_at++].val.clusterDim.z = 1;
  }
  if (pdl_mask() & kPdlHook) {
    at[n_at].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n_at++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = at;
  cfg.numAttrs = n_at;
  return cudaLaunchKernelEx(&cfg, linear_int_kernel<OutT, NT, kMode>, tw, tx, g.scale, g.w_scale, g.bias, g.offsets, g.n_rows, g.K, g.N, g.E,
                            p.tile_tok, p.parts, static_cast<OutT*>(g.out), g.ld_out, vec, g_i8_test_stall.load(std::memory_order_relaxed));
}

// A k-block of a tile of n tokens costs a CTA max(2 n, 256 + n) clocks in a pair and 256 + 2 n alone: the instructions take 2 n, and
// shared memory moves each operand byte twice at 128 bytes a clock.  What a tile costs beside its k-blocks is some 1500 clocks, in
// a pair 3000, and 2500 + 60 n more where its parts have to meet.  Among tiles of 32, 64 and 128 tokens, in parts or not, and pairs
// of 256 the one is taken whose waves cost least.  (16 x 4096 codes by 4096 channels: in four parts 8.4 us, 9.7 in one; 16 x 14336:
// 14.9 and 24.5; 128 x 4096 by 4096 in tiles of 32: 7.9 us.  Pairs of smaller tiles, which fit the waves better by this count, were
// slower: 256 x 4096 by 4096 10.2 us in pairs of 64 tokens, 8.6 in single tiles of 64; 1000 x 5120 by 9992 no faster with 5 x 200
// tokens than with 4 x 250.)
// By experts the host knows the rows' average alone, and a tile costs little more than the tokens it has: tiles hold about twice an
// even share, in pairs above 96.  (64 experts of 2048 x 2048, 32 rows each on average: 48.4 us with tiles of 32 tokens, 44.1 with 64;
// 64 rows: 50.3 with 64, 45.5 with 128; 128 rows: 62.9 with 128, 55.2 in pairs.  8 experts of 4096 x 4096, 24 rows: 22.2 with 32, 24.7
// with 64; 96 rows: 26.0 with 128, 26.9 in pairs.)
TilePlan tile_plan(const Gemm& g, int n_sms) {
  const long long kbs = div_up(g.K, kKBytes);
  TilePlan best = {kSingle, 32, 32, 1};
  double least = 1e30;
  const auto consider = [&](int mode, int nt, int tile_tok, int parts) {
    const long long tiles = tiles_at_most(g, tile_tok, mode == kPairs ? 2 * kTileCh : kTileCh);
    if (parts > 1 && (tiles * parts > n_sms || kbs < 4 * parts)) return;
    const long long waves = parts > 1 ? 1 : div_up(tiles, mode == kPairs ? n_sms / 2 : n_sms);
    const long long n = div_up(g.n_rows, div_up(g.n_rows, tile_tok)), a = mode == kPairs ? (2 * n > 256 + n ? 2 * n : 256 + n) : 256 + 2 * n;
    const double cost = (double)waves * (double)(div_up(kbs, parts) * a + (parts > 1 ? 4000 + 60 * n : (mode == kPairs ? 3000 : 1500)));
    if (cost < least) {
      least = cost;
      best = TilePlan{mode, nt, tile_tok, parts};
    }
  };
  if (g.E == 1) {
    for (int nt = 32; nt <= 128; nt *= 2)
      for (int parts = 1; parts <= kMostParts; parts *= 2) consider(parts > 1 ? kSplit : kSingle, nt, nt, parts);
    consider(kPairs, 256, 256, 1);
    return best;
  }
  const int even = (int)div_up(g.n_rows, g.E);
  if (even > 96) return TilePlan{kPairs, 256, 256, 1};
  const int nt = even <= 24 ? 32 : (even <= 40 ? 64 : 128);
  for (int parts = 1; parts <= kMostParts; parts *= 2) consider(parts > 1 ? kSplit : kSingle, nt, nt, parts);
  return best;
}

template <typename OutT>
cudaError_t gemm_pick(const Gemm& g, int dev, int n_sms, cudaStream_t s) {
  const TilePlan p = tile_plan(g, n_sms);
  if (p.mode == kPairs) return gemm_launch<OutT, 256, kPairs>(g, p, dev, n_sms, s);
  if (p.mode == kSplit)
    return p.nt == 32 ? gemm_launch<OutT, 32, kSplit>(g, p, dev, n_sms, s)
                      : (p.nt == 64 ? gemm_launch<OutT, 64, kSplit>(g, p, dev, n_sms, s) : gemm_launch<OutT, 128, kSplit>(g, p, dev, n_sms, s));
  return p.nt == 32 ? gemm_launch<OutT, 32, kSingle>(g, p, dev, n_sms, s)
                    : (p.nt == 64 ? gemm_launch<OutT, 64, kSingle>(g, p, dev, n_sms, s) : gemm_launch<OutT, 128, kSingle>(g, p, dev, n_sms, s));
}

int gemm_call(const Gemm& g, int dtype, void* stream, char* errbuf, int errbuf_len) {
  if (op_elem_size(dtype) == 0) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "dtype %d is no MIX_DTYPE_*", dtype);
  if (g.n_rows < 0 || g.n_rows > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "%d rows, outside [0, %d]", g.n_rows, kOpMaxRows);
  if (g.K < 16 || g.K > MIX_I8_MAX_K) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "K %d outside [16, %d]", g.K, MIX_I8_MAX_K);
  if (g.K % 16) MIX_OP_FAIL(MIX_ERR_UNSUPPORTED, "K %d is not a multiple of 16", g.K);
  if (g.N < 1) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "N %d is below 1", g.N);
  if (g.E < 1 || g.E > kOpMaxExperts) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n_experts %d outside [1, %d]", g.E, kOpMaxExperts);
  if ((long long)g.E * g.N > 0x7fffff00ll) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "%lld rows of W", (long long)g.E * g.N);
  const long long tiles = ((long long)g.n_rows / 32 + g.E) * ((g.N + kTileCh - 1) / kTileCh);
  if (tiles > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n_rows %d x N %d has too many tiles", g.n_rows, g.N);
  if (g.ld_out < g.N) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row stride %lld of the output is below N %d", g.ld_out, g.N);
  if (g.n_rows == 0) return MIX_OK;
  if (!g.codes || !g.scale || !g.w || !g.w_scale || !g.out) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "codes, scale, W, w_scale and out are required");
  if (((uintptr_t)g.codes | (uintptr_t)g.w) & 15u) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "codes and W must be 16-byte aligned");
  int dev, n_sms;
  MIX_OP_CUDA(op_device(&dev, &n_sms));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MIX_DTYPE_F32) MIX_OP_CUDA(gemm_pick<float>(g, dev, n_sms, s));
  else if (dtype == MIX_DTYPE_BF16) MIX_OP_CUDA(gemm_pick<__nv_bfloat16>(g, dev, n_sms, s));
  else MIX_OP_CUDA(gemm_pick<__half>(g, dev, n_sms, s));
  return MIX_OK;
}

template <typename T, bool vec>
cudaError_t quantize_launch_as(const void* x, long long ld, int x_rows, const int* order, int div, int n_rows, int d, signed char* codes,
                               float* scale, cudaStream_t s) {
  const T* xt = static_cast<const T*>(x);
  if (d <= 1024)                                               // a warp holds the row
    return launch_pdl(kPdlHook, quantize_rows_kernel<T, 32, vec>, dim3((unsigned)((n_rows + 3ll) / 4)), dim3(128), 0, s, xt, ld, x_rows, order, div,
                      n_rows, d, codes, scale);
  if (d <= 4096)
    return launch_pdl(kPdlHook, quantize_rows_kernel<T, 128, vec>, dim3((unsigned)n_rows), dim3(128), 0, s, xt, ld, x_rows, order, div, n_rows, d,
                      codes, scale);
  return launch_pdl(kPdlHook, quantize_rows_kernel<T, 256, vec>, dim3((unsigned)n_rows), dim3(256), 0, s, xt, ld, x_rows, order, div, n_rows, d,
                    codes, scale);
}
template <typename T>
cudaError_t quantize_launch(const void* x, long long ld, int x_rows, const int* order, int div, int n_rows, int d, signed char* codes,
                            float* scale, cudaStream_t s) {
  const int vec = (((uintptr_t)x | (uintptr_t)(ld * 2)) & 15u) == 0;
  return vec ? quantize_launch_as<T, true>(x, ld, x_rows, order, div, n_rows, d, codes, scale, s)
             : quantize_launch_as<T, false>(x, ld, x_rows, order, div, n_rows, d, codes, scale, s);
}

template <typename T, bool vec>
cudaError_t combine_launch_as(const void* y, long long ld_y, int y_rows, const float* weights, const int* position, int T_rows, int k, int N,
                              void* out, long long ld_out, cudaStream_t s) {
  constexpr int kCols = kCombineThreads * (vec ? RowVec<T>::VW : 1);
  const dim3 grid((unsigned)T_rows, (unsigned)((N + kCols - 1) / kCols));
#define MIX_COMBINE(K)                                                                                                                \
  return launch_pdl(kPdlHook, combine_kernel<T, K, vec>, grid, dim3(kCombineThreads), 0, s, static_cast<const T*>(y), ld_y, y_rows, weights, \
                    position, k, N, static_cast<T*>(out), ld_out)
  if (k <= 2) MIX_COMBINE(2);
  if (k <= 4) MIX_COMBINE(4);
  if (k <= 8) MIX_COMBINE(8);
  MIX_COMBINE(kOpMaxTopk);
#undef MIX_COMBINE
}
template <typename T>
cudaError_t combine_launch(const void* y, long long ld_y, int y_rows, const float* weights, const int* position, int T_rows, int k, int N,
                           void* out, long long ld_out, cudaStream_t s) {
  const bool vec = (((uintptr_t)y | (uintptr_t)out | (uintptr_t)(ld_y * (long long)sizeof(T)) | (uintptr_t)(ld_out * (long long)sizeof(T))) & 15u) == 0;
  return vec ? combine_launch_as<T, true>(y, ld_y, y_rows, weights, position, T_rows, k, N, out, ld_out, s)
             : combine_launch_as<T, false>(y, ld_y, y_rows, weights, position, T_rows, k, N, out, ld_out, s);
}

template <typename T, bool vec>
cudaError_t combine_grad_launch_as(const void* y, long long ld_y, int y_rows, const float* weights, const int* position, int T_rows, int k, int N,
                                   const void* d_out, long long ld_d, float* d_weights, void* d_y, long long ld_dy, cudaStream_t s) {
#define MIX_COMBINE_GRAD(K)                                                                                                                   \
  return launch_pdl(kPdlHook, combine_grad_kernel<T, K, vec>, dim3((unsigned)T_rows), dim3(kCombineGradThreads), 0, s, static_cast<const T*>(y), ld_y, \
                    y_rows, weights, position, k, N, static_cast<const T*>(d_out), ld_d, d_weights, static_cast<T*>(d_y), ld_dy)
  if (k <= 2) MIX_COMBINE_GRAD(2);
  if (k <= 8) MIX_COMBINE_GRAD(8);
  MIX_COMBINE_GRAD(kOpMaxTopk);
#undef MIX_COMBINE_GRAD
}
template <typename T>
cudaError_t combine_grad_launch(const void* y, long long ld_y, int y_rows, const float* weights, const int* position, int T_rows, int k, int N,
                                const void* d_out, long long ld_d, float* d_weights, void* d_y, long long ld_dy, cudaStream_t s) {
  const long long es = sizeof(T);
  const bool vec = (((uintptr_t)y | (uintptr_t)d_out | (uintptr_t)d_y | (uintptr_t)(ld_y * es) | (uintptr_t)(ld_d * es) | (uintptr_t)(d_y ? ld_dy * es : 0)) & 15u) == 0;
  return vec ? combine_grad_launch_as<T, true>(y, ld_y, y_rows, weights, position, T_rows, k, N, d_out, ld_d, d_weights, d_y, ld_dy, s)
             : combine_grad_launch_as<T, false>(y, ld_y, y_rows, weights, position, T_rows, k, N, d_out, ld_d, d_weights, d_y, ld_dy, s);
}

}  // namespace

extern "C" int mix_quantize_rows(const void* x, int dtype, long long ld, int x_rows, const int* order, int k, int n_rows, int d,
                                    signed char* codes, float* scale, void* stream, char* errbuf, int errbuf_len) {
  if (dtype != MIX_DTYPE_BF16 && dtype != MIX_DTYPE_F16) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "dtype %d is neither bf16 nor fp16", dtype);
  if (n_rows < 0 || x_rows < 0 || n_rows > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "%d rows of %d", n_rows, x_rows);
  if (d < 16 || d > MIX_I8_MAX_K) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "d %d outside [16, %d]", d, MIX_I8_MAX_K);
  if (d % 16) MIX_OP_FAIL(MIX_ERR_UNSUPPORTED, "d %d is not a multiple of 16", d);
  if (ld < d) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row stride %lld is below d %d", ld, d);
  if (order && k < 1) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "k %d is below 1", k);
  if (!order && n_rows != x_rows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "without an order the %d rows of x make as many, not %d", x_rows, n_rows);
  if (n_rows == 0) return MIX_OK;
  if ((!x && x_rows > 0) || !codes || !scale) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "x, codes and scale are required");
  if ((uintptr_t)codes & 15u) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MIX_DTYPE_BF16) MIX_OP_CUDA(quantize_launch<__nv_bfloat16>(x, ld, x_rows, order, k, n_rows, d, codes, scale, s));
  else MIX_OP_CUDA(quantize_launch<__half>(x, ld, x_rows, order, k, n_rows, d, codes, scale, s));
  return MIX_OK;
}

extern "C" int mix_linear_int(const signed char* codes, const float* scale, int T, int K, const signed char* W, const float* w_scale, int N,
                             const float* bias, void* out, int out_dtype, long long ld_out, void* stream, char* errbuf, int errbuf_len) {
  return gemm_call(Gemm{codes, scale, W, w_scale, bias, nullptr, T, K, N, 1, out, ld_out}, out_dtype, stream, errbuf, errbuf_len);
}

extern "C" int mix_linear_int_grouped(const signed char* codes, const float* scale, int n_rows, int K, const signed char* W, const float* w_scale,
                                     int n_experts, int N, const int* offsets, const float* bias, void* out, int out_dtype, long long ld_out,
                                     void* stream, char* errbuf, int errbuf_len) {
  if (!offsets) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "offsets is NULL");
  return gemm_call(Gemm{codes, scale, W, w_scale, bias, offsets, n_rows, K, N, n_experts, out, ld_out}, out_dtype, stream, errbuf, errbuf_len);
}

extern "C" int mix_debug_linear_int_stall(int on) { return g_i8_test_stall.exchange(on != 0); }

extern "C" int mix_linear_int_status(unsigned* bits, void* stream, char* errbuf, int errbuf_len) {
  if (!bits) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "bits is NULL");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaStreamCaptureStatus capture;
  MIX_OP_CUDA(cudaStreamIsCapturing(s, &capture));
  if (capture != cudaStreamCaptureStatusNone) MIX_OP_FAIL(MIX_ERR_UNSUPPORTED, "the status cannot be read in a capture");   // (which goes on)
  // Read first, cleared only where something was found: what a product on another stream raises in between is the same bit, which this
  // call reports.  Copy and clearing one behind the other lost it.
  const unsigned zero = 0;
  unsigned found = 0;
  MIX_OP_CUDA(cudaMemcpyFromSymbolAsync(&found, g_i8_status, sizeof(unsigned), 0, cudaMemcpyDeviceToHost, s));
  MIX_OP_CUDA(cudaStreamSynchronize(s));
  if (found) {
    MIX_OP_CUDA(cudaMemcpyToSymbolAsync(g_i8_status, &zero, sizeof(unsigned), 0, cudaMemcpyHostToDevice, s));
    MIX_OP_CUDA(cudaStreamSynchronize(s));
  }
  *bits = found;
  return MIX_OK;
}

extern "C" int mix_expert_combine(const void* y, int dtype, long long ld_y, int y_rows, const float* weights, const int* position, int T, int k,
                                  int N, void* out, long long ld_out, void* stream, char* errbuf, int errbuf_len) {
  if (op_elem_size(dtype) == 0) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "dtype %d is no MIX_DTYPE_*", dtype);
  if (T < 0 || y_rows < 0 || T > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "%d tokens, %d rows of y", T, y_rows);
  if (k < 1 || k > kOpMaxTopk) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "k %d outside [1, %d]", k, kOpMaxTopk);
  if (N < 1 || N > MIX_COMBINE_MAX_N) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "N %d outside [1, %d]", N, MIX_COMBINE_MAX_N);
  if (ld_y < N || ld_out < N) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row strides %lld, %lld below N %d", ld_y, ld_out, N);
  if (T == 0) return MIX_OK;
  if ((!y && y_rows > 0) || !weights || !position || !out) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "y, weights, position and out are required");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MIX_DTYPE_F32) MIX_OP_CUDA(combine_launch<float>(y, ld_y, y_rows, weights, position, T, k, N, out, ld_out, s));
  else if (dtype == MIX_DTYPE_BF16) MIX_OP_CUDA(combine_launch<__nv_bfloat16>(y, ld_y, y_rows, weights, position, T, k, N, out, ld_out, s));
  else MIX_OP_CUDA(combine_launch<__half>(y, ld_y, y_rows, weights, position, T, k, N, out, ld_out, s));
  return MIX_OK;
}

extern "C" int mix_expert_combine_grad(const void* y, int dtype, long long ld_y, int y_rows, const float* weights, const int* position, int T, int k,
                                       int N, const void* d_out, long long ld_d, float* d_weights, void* d_y, long long ld_dy, void* stream,
                                       char* errbuf, int errbuf_len) {
  if (op_elem_size(dtype) == 0) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "dtype %d is no MIX_DTYPE_*", dtype);
  if (T < 0 || y_rows < 0 || T > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "%d tokens, %d rows of y", T, y_rows);
  if (k < 1 || k > kOpMaxTopk) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "k %d outside [1, %d]", k, kOpMaxTopk);
  if (N < 1 || N > MIX_COMBINE_MAX_N) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "N %d outside [1, %d]", N, MIX_COMBINE_MAX_N);
  if (ld_y < N || ld_d < N || (d_y && ld_dy < N)) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row strides %lld, %lld, %lld below N %d", ld_y, ld_d, ld_dy, N);
  if (T == 0) return MIX_OK;
  if ((!y && y_rows > 0) || !position || !d_out || !d_weights || (d_y && !weights))
    MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "y, position, d_out, d_weights (and weights for d_y) are required");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MIX_DTYPE_F32) MIX_OP_CUDA(combine_grad_launch<float>(y, ld_y, y_rows, weights, position, T, k, N, d_out, ld_d, d_weights, d_y, ld_dy, s));
  else if (dtype == MIX_DTYPE_BF16)
    MIX_OP_CUDA(combine_grad_launch<__nv_bfloat16>(y, ld_y, y_rows, weights, position, T, k, N, d_out, ld_d, d_weights, d_y, ld_dy, s));
  else MIX_OP_CUDA(combine_grad_launch<__half>(y, ld_y, y_rows, weights, position, T, k, N, d_out, ld_d, d_weights, d_y, ld_dy, s));
  return MIX_OK;
}

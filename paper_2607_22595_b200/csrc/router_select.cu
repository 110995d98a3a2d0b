// The selection behind the router: the k experts of a token with their weights, the gradient of those weights, and the
// tokens sorted by expert.
//
//   router_topk_kernel       idx[t, :] = the k largest logits of row t, largest first, the lower index first among equal ones;
//                            w = p[idx] or p[idx] / sum of the chosen, p = softmax or sigmoid of the row.
//   router_topk_grad_kernel  d_logits of sum_j d_w[t, j] w[t, j].
//   expert_hist_kernel,      a stable counting sort of the flat entries (t, j) by expert.
//   expert_order_kernel
//
// All three are streams over [T, E] or [T, k]; a row sits in the registers of G = E / 8 lanes, so that a warp holds
// 32 / G rows and every load is one 16-byte vector.
#include "op_common.cuh"
#include "tc_common.cuh"

using namespace mix;

namespace {

constexpr int kSelThreads = 256;

// ---------------------------------------------------------------------------------------------------- selection
// The selection compares the logits themselves, never probabilities: those round, and two logits that differ could tie.
//
// What bounds it is comparisons and selections, which issue at half rate, so it compares keys that carry the column: the logit's
// order-preserving bits, the lowest 3 to 9 replaced by ~column.  No two keys of a row are equal, and a round is one reduction over
// the G lanes.  fp32 logits lose bits by that: where two neighbours among the first k + 1 agree in what is left, the row is done
// again by rounds that compare logits and columns (16-bit logits lose none).
// Rows of up to 64 experts: k rounds over all keys, 32 / G rows of a warp side by side.
// Wider rows: a lane keeps its three largest keys; one that has given its first offers its second.  Where a lane gave all three and
// has more above the last key (8 of 256: four rows in a thousand) the row is done again too.
// 65536 rows of 256 fp32, k = 8: 29.8 us with the weights renormalised, 32.5 with the softmax over the row (76 by rounds over logits); the logits' stream
// alone takes 10.3.  That is of logits that hardly ever tie.  fp32 logits that hold bf16 values, a bf16 router's after steering, tie in a third
// to a half of the warps, which are done again: 44.7 and 47.5 us, 31.8 instead of 19.5 for rows of 128, 17.4 instead of 11.7 for rows
// of 64 (k = 6).  The same logits in bf16 lose no bits: 28.6 and 31.3 us, 17.4, 10.3.
template <int G>
__device__ __forceinline__ unsigned group_max_key(unsigned x) {
  if (G == 32) return __reduce_max_sync(0xffffffffu, x);
#pragma unroll
  for (int o = 1; o < G; o <<= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
template <typename T, int G, int V>
__global__ void __launch_bounds__(kSelThreads)
router_topk_kernel(const T* __restrict__ logits, long long ld, int vec, int T_rows, int E, int k, int act, int renorm,
                   const int* __restrict__ n_live, int* __restrict__ idx, float* __restrict__ weights) {
  constexpr int S = G >= kOpMaxTopk ? 1 : (G == 1 ? 8 : kOpMaxTopk / G);   // chosen entries a lane keeps: entry j is lane j % G's
  pdl_wait();
  pdl_launch_dependents();
  const int sub = threadIdx.x & (G - 1);
  const int live = n_live ? min(*n_live, T_rows) : T_rows;
  const long long t = ((long long)blockIdx.x * kSelThreads + threadIdx.x) / G;
  float x[V];
  if (t < live) {
    load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = -INFINITY;
  }
  float sum = 0.f;                                                         // a NaN is never chosen; one that is there makes the sum one
#pragma unroll
  for (int v = 0; v < V; ++v) sum += x[v];
  if (__any_sync(0xffffffffu, sum != sum)) {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = fmaxf(x[v], -INFINITY);             // (the larger of a NaN and a number is the number)
  }
  constexpr unsigned kCol = G * V - 1;                                     // the key's bits that hold ~column
  constexpr unsigned kNone = 0x007fffffu & ~kCol;                          // -inf's key
  constexpr int kRounds = G == 1 ? 8 : kOpMaxTopk;
  static_assert((kCol & G * V) == 0, "a power of two");
  unsigned key[V], mine[S];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const unsigned bits = __float_as_uint(x[v] + 0.f);                     // -0 and 0 are equal
    key[v] = ((bits ^ ((unsigned)((int)bits >> 31) | 0x80000000u)) & ~kCol) | (kCol - (unsigned)row_col<T, G>(v, sub));
  }
#pragma unroll
  for (int s = 0; s < S; ++s) mine[s] = 0u;
  const int n_rounds = sizeof(T) == 4 ? k + 1 : k;
  bool unsure = false;
  if (S == 1) {
    unsigned k1[V / 2], k2[V / 2], k3[V / 4];                              // sorted parts of the lane's keys, their three largest
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      k1[i] = max(key[2 * i], key[2 * i + 1]);
      k2[i] = min(key[2 * i], key[2 * i + 1]);
    }
#pragma unroll
    for (int n = V / 4; n > 0; n /= 2) {
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const unsigned m = min(k1[i], k1[i + n]), l = max(k2[i], k2[i + n]);
        k1[i] = max(k1[i], k1[i + n]);
        k2[i] = max(m, l);
        k3[i] = n == V / 4 ? min(m, l) : max(min(m, l), max(k3[i], k3[i + n]));
      }
    }
    unsigned first = k1[0], second = k2[0], third = k3[0], last = 0u;
#pragma unroll
    for (int j = 0; j < kRounds + 1; ++j) {
      if (j >= n_rounds) break;
      last = group_max_key<G>(first);
      mine[0] = j == sub ? last : mine[0];
      const bool mine_goes = first == last;
      first = mine_goes ? second : first;
      second = mine_goes ? third : second;
      third = mine_goes ? 0u : third;
    }
    if (__any_sync(0xffffffffu, first == 0u)) {                            // a lane gave all three
      int above = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) above += key[v] >= last;
      unsure = first == 0u && above > 3;
    }
    unsigned after = __shfl_down_sync(0xffffffffu, mine[0], 1, G);         // (by all lanes)
    if (sub == k - 1) after = last;                                        // of the round behind the last one chosen
    if (sizeof(T) == 4) unsure |= sub < k && (mine[0] & ~kCol) > kNone && ((after ^ mine[0]) & ~kCol) == 0u;
  } else {
    unsigned before = 0u;
#pragma unroll
    for (int j = 0; j < kRounds + 1; ++j) {
      if (j >= n_rounds) break;
      unsigned m = key[0];
#pragma unroll
      for (int v = 1; v < V; ++v) m = max(m, key[v]);
      m = group_max_key<G>(m);
      if (j < kRounds && j % G == sub) mine[j < kRounds ? j / G : 0] = m;
      if (sizeof(T) == 4) unsure |= (m & ~kCol) > kNone && ((m ^ before) & ~kCol) == 0u;
      before = m;
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = key[v] == m ? 0u : key[v];
    }
  }
  const bool rounds = __any_sync(0xffffffffu, unsure);
  int my_idx[S];
  float my_x[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const bool some = !rounds && s * G + sub < k && (mine[s] & ~kCol) > kNone;
    my_idx[s] = some ? (int)(kCol - (mine[s] & kCol)) : -1;
    my_x[s] = -INFINITY;
    // (the bits that gave way to the column were 0 in a 16-bit logit, 1 in the key of a negative one)
    if (some) my_x[s] = sizeof(T) == 4 ? to_f32(logits[t * ld + my_idx[s]]) : key2f((mine[s] & 0x80000000u) ? mine[s] & ~kCol : mine[s] | kCol);
  }
  if (rounds) {
    float left[V];
#pragma unroll
    for (int v = 0; v < V; ++v) left[v] = x[v];
#pragma unroll
    for (int j = 0; j < kRounds; ++j) {
      if (j >= k) break;
      const float m = group_max<G>(top_of<V>(left));
      unsigned c = 0xffffffffu;
#pragma unroll
      for (int v = V - 1; v >= 0; --v) c = left[v] == m ? (unsigned)row_col<T, G>(v, sub) : c;   // (columns rise with v)
      if (G == 32) {
        c = __reduce_min_sync(0xffffffffu, c);
      } else {
#pragma unroll
        for (int o = 1; o < G; o <<= 1) c = min(c, __shfl_xor_sync(0xffffffffu, c, o));
      }
#pragma unroll
      for (int v = 0; v < V; ++v) left[v] = (unsigned)row_col<T, G>(v, sub) == c ? -INFINITY : left[v];
      if (j % G == sub && m > -INFINITY) {
        my_idx[j / G] = (int)c;
        my_x[j / G] = m;
      }
    }
  }
  const float top = __shfl_sync(0xffffffffu, my_x[0], 0, G);               // the first one chosen
  const bool plain = act == MIX_ACT_SIGMOID && !renorm;                    // the weight is the sigmoid itself
  float total = 0.f;
  if (act == MIX_ACT_SOFTMAX && !renorm) total = scores<V>(act, top, false, x);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    my_x[s] = my_idx[s] < 0 ? 0.f : (plain ? sigmoid_row(my_x[s]) : score(act, my_x[s], top));
    if (renorm) total += my_x[s];
  }
  if (!plain) total = group_sum<G>(total);
  const float norm = plain ? 1.f : total;                                  // (divided: the weight of a single one chosen is 1 and its gradient 0)
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int j = s * G + sub;
    if (j < k && t < T_rows) {
      idx[t * k + j] = my_idx[s];
      weights[t * k + j] = my_idx[s] >= 0 ? __fdiv_rn(my_x[s], norm) : 0.f;
    }
  }
}

// ---------------------------------------------------------------------------------------------------- gradient
// With w the weights that the selection gave, g = d_w at the entries that name an expert, and s = sum_j g_j w_j:
//   softmax, renormalised  dx_i = w_i (g_i - s)                 at the chosen experts, 0 elsewhere
//   softmax                dx_c = p_c (g_c - s)                 for every expert c, g_c = 0 where it was not chosen
//   sigmoid                dx_i = w_i (1 - sigmoid(x_i)) g_i    at the chosen experts
//   sigmoid, renormalised  dx_i = w_i (1 - sigmoid(x_i)) (g_i - s)
// Entries without an expert are not read further: what stands in their d_w (NaN, say) does not matter.
//
// Where a lane has one chosen entry (more than 64 experts) the row is written as if nothing had been chosen -- p (-s), or zeros --
// and the lanes then write their own entries over it, w (g - s): w is p there.  Narrower rows compare each entry with each
// column of a lane, for 32 / G rows at a time.  65536 rows of 256: 38 us with the entries spread over the row in shared memory,
// 22.7 so (5.9 TB/s); reading and writing the logits alone takes 20.6.
template <typename T, int G, int V>
__global__ void __launch_bounds__(kSelThreads)
router_topk_grad_kernel(const T* __restrict__ logits, long long ld, int vec, int T_rows, int E, int k, int act, int renorm,
                        const int* __restrict__ idx, const float* __restrict__ weights, const float* __restrict__ d_weights,
                        T* __restrict__ d_logits, long long ld_d, int vec_d) {
  constexpr int S = G >= kOpMaxTopk ? 1 : (G == 1 ? 8 : kOpMaxTopk / G);
  pdl_wait();
  pdl_launch_dependents();
  const int sub = threadIdx.x & (G - 1), lane = threadIdx.x & 31;
  const long long t = ((long long)blockIdx.x * kSelThreads + threadIdx.x) / G;
  const bool row = t < T_rows, dense = act == MIX_ACT_SOFTMAX && !renorm;
  float p[V];
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = -INFINITY;
  if (dense && row) load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, p);
  int my_idx[S];
  float my_g[S], my_w[S];
#pragma unroll
  for (int i = 0; i < S; ++i) {
    const int j = i * G + sub;
    const bool in = row && j < k;
    my_idx[i] = in ? idx[t * k + j] : -1;
    my_g[i] = in ? d_weights[t * k + j] : 0.f;
    my_w[i] = in ? weights[t * k + j] : 0.f;
  }
  float s = 0.f;
  bool any = false;
#pragma unroll
  for (int i = 0; i < S; ++i) {
    const bool ok = (unsigned)my_idx[i] < (unsigned)E;
    if (!ok) {
      my_idx[i] = -1;
      my_g[i] = my_w[i] = 0.f;
    }
    s += my_g[i] * my_w[i];
    any |= ok;
  }
  s = group_sum<G>(s);
  float d[V];
#pragma unroll
  for (int v = 0; v < V; ++v) d[v] = 0.f;
  if (dense) {
    any = group_any<G>(any);
    const float total = group_sum<G>(scores<V>(act, group_max<G>(top_of<V>(p)), false, p));
    const float inv = any && total > 0.f ? rcp_hw(total) : 0.f;
    const float less = S == 1 ? inv * -s : inv;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p[v] *= less;
      if (S == 1) d[v] = p[v];
    }
  } else {
#pragma unroll
    for (int i = 0; i < S; ++i) {                                // the factors that g is multiplied with, and what is taken off it
      if (act == MIX_ACT_SIGMOID && my_idx[i] >= 0) my_w[i] *= sigmoid_row(-to_f32(logits[t * ld + my_idx[i]]));
    }
    if (act == MIX_ACT_SIGMOID && !renorm) s = 0.f;
  }
  if (S == 1) {
    if (row) store_row<T, G, V>(d_logits + t * ld_d, E, sub, vec_d != 0, d);
    // the same expert twice in a row (never in what the selection gives): of a dense row its entries share one -s
    const unsigned same = __match_any_sync(0xffffffffu, my_idx[0] < 0 ? -1 : my_idx[0] + (lane / G) * kOpMaxExperts);
    float mine = my_w[0] * (my_g[0] - s);
    if (__any_sync(0xffffffffu, my_idx[0] >= 0 && (same & (same - 1u)) != 0u)) {
      const float part = dense ? my_w[0] * my_g[0] : mine;
      mine = dense ? my_w[0] * -s : 0.f;
      for (int i = 0; i < 32; ++i) {
        const float other = __shfl_sync(0xffffffffu, part, i);
        if ((same >> i) & 1u) mine += other;
      }
    }
    __syncwarp();                                                // the row lies below the entries
    if (my_idx[0] >= 0 && lane == __ffs(same) - 1) d_logits[t * ld_d + my_idx[0]] = from_f32<T>(mine);
  } else {
#pragma unroll
    for (int j = 0; j < (G == 1 ? 8 : kOpMaxTopk); ++j) {
      if (j >= k) break;
      const int at = __shfl_sync(0xffffffffu, my_idx[j / G], j % G, G);
      const float g = __shfl_sync(0xffffffffu, dense ? my_g[j / G] : my_w[j / G] * (my_g[j / G] - s), j % G, G);
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] += row_col<T, G>(v, sub) == at ? g : 0.f;
    }
    if (dense) {
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] = p[v] * (d[v] - s);
    }
    if (row) store_row<T, G, V>(d_logits + t * ld_d, E, sub, vec_d != 0, d);
  }
}

// ---------------------------------------------------------------------------------------------------- order by expert
constexpr int kOrdThreads = 512;
constexpr int kOrdWarps = kOrdThreads / 32;
constexpr int kOrdSteps = 4;                                    // entries a lane takes
constexpr int kOrdChunk = kOrdThreads * kOrdSteps;              // entries a CTA takes, at most
constexpr int kOrdBuckets = kOpMaxExperts + 1;                  // the last of a call's holds the entries without an expert
constexpr int kOrdCluster = 8;                                  // CTAs that can look into each other's counts
static_assert(kOrdChunk <= 65535, "places within a chunk in 16 bits");

__host__ __device__ constexpr int hist_stride(int E) { return (E + 1 + 3) & ~3; }   // counts of a chunk, in whole 16-byte vectors
__device__ __forceinline__ int bucket_of(int i, int E) { return (unsigned)i < (unsigned)E ? i : E; }

__global__ void __launch_bounds__(kOrdThreads)
expert_hist_kernel(const int* __restrict__ idx, int n, int E, int steps, int* __restrict__ hist) {
  __shared__ int h[kOrdBuckets];
  pdl_wait();
  pdl_launch_dependents();
  const int threads = blockDim.x, base = blockIdx.x * threads * steps;
  int e[kOrdSteps];
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * threads + threadIdx.x;
    e[i] = i < steps && at < n ? bucket_of(idx[at], E) : -1;
  }
  for (int i = threadIdx.x; i <= E; i += threads) h[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i)
    if (e[i] >= 0) atomicAdd(&h[e[i]], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < hist_stride(E); i += threads) hist[(size_t)blockIdx.x * hist_stride(E) + i] = i <= E ? h[i] : 0;
}

// For many chunks: the counts of a chunk become those of the chunks in front of it, in place; the row behind the last chunk receives
// the sums over all.  A CTA has 32 buckets, a thread every bucket's chunks of one of 32 stretches.
constexpr int kScanThreads = 1024;
__global__ void __launch_bounds__(kScanThreads)
expert_scan_kernel(int* __restrict__ hist, int n_chunks, int stride) {
  __shared__ int part[kScanThreads / 32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  const int each = (n_chunks + kScanThreads / 32 - 1) / (kScanThreads / 32), c0 = min(n_chunks, r * each), c1 = min(n_chunks, c0 + each);
  int sum = 0;
  if (b < stride) {
#pragma unroll 8
    for (int c = c0; c < c1; ++c) sum += hist[(size_t)c * stride + b];
  }
  part[r][threadIdx.x & 31] = sum;
  __syncthreads();
  if (r == 0) {
    int run = 0;
#pragma unroll
    for (int i = 0; i < kScanThreads / 32; ++i) {
      const int v = part[i][threadIdx.x];
      part[i][threadIdx.x] = run;
      run += v;
    }
    if (b < stride) hist[(size_t)n_chunks * stride + b] = run;
  }
  __syncthreads();
  if (b < stride) {
    int run = part[r][threadIdx.x & 31];
    for (int c = c0; c < c1; c += 8) {
      int v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < c1 ? hist[(size_t)(c + i) * stride + b] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i < c1) hist[(size_t)(c + i) * stride + b] = run;
        run += v[i];
      }
    }
  }
}

// Entry i of the CTA's chunk goes to  (entries of lower experts) + (entries of this expert in earlier chunks, in earlier warps
// of the CTA, earlier in the warp).  The counts of the other chunks: up to eight chunks are one cluster, whose CTAs read them from
// each other's shared memory -- a call of up to 16384 entries is this one launch -- beyond that they are expert_hist_kernel's, and
// of more than 64 chunks summed up by expert_scan_kernel.
// A chunk is sorted in shared memory and leaves expert by expert: written straight from the registers every entry of a warp goes to
// another line, which took an SM 8192 turns, half of the kernel's time.
// A warp takes `steps` times 32 entries, the last warps of a call's last chunk fewer.
struct OrderShared {
  int before[kOrdBuckets + 3], start[kOrdBuckets + 3], mine[kOrdBuckets + 3], total[kOrdBuckets + 3];
  int warp_sum[kOrdWarps];
  unsigned short warp_count[kOrdWarps][kOrdBuckets + 1];        // (an even number of them: rows on 4 bytes)
  unsigned sorted[kOrdChunk];                                   // place in the chunk | expert << 16
};
template <bool kCluster>
__global__ void __launch_bounds__(kOrdThreads)
expert_order_kernel(const int* __restrict__ idx, int n, int E, const int* __restrict__ hist, int n_chunks, int steps, int scanned, int* __restrict__ offsets,
                    int* __restrict__ order, int* __restrict__ position) {
  extern __shared__ __align__(16) unsigned char order_smem[];
  OrderShared* sh = reinterpret_cast<OrderShared*>(order_smem);
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
  const int chunk = blockIdx.x * (int)blockDim.x * steps, in_chunk = min(n - chunk, (int)blockDim.x * steps);
  const int base = warp * 32 * steps;
  int bucket[kOrdSteps], rank[kOrdSteps];
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * 32 + lane;
    bucket[i] = i < steps && at < in_chunk ? bucket_of(idx[chunk + at], E) : E + 1;
  }
  for (int e = lane; e < (E + 2) / 2; e += 32) reinterpret_cast<unsigned*>(sh->warp_count[warp])[e] = 0u;
  for (int e = threadIdx.x; e <= E; e += blockDim.x) sh->total[e] = sh->before[e] = 0;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    if (i >= steps || base + i * 32 >= in_chunk) break;
    // the lanes with the same bucket, bit by bit (a match instruction takes a turn per value in the warp)
    unsigned same = 0xffffffffu;
    for (int bit = 1; bit <= E + 1; bit <<= 1) {
      const unsigned with = __ballot_sync(0xffffffffu, (bucket[i] & bit) != 0);
      same &= (bucket[i] & bit) != 0 ? with : ~with;
    }
    const int first = __ffs(same) - 1;
    int old = 0;
    if (lane == first && bucket[i] <= E) {
      old = sh->warp_count[warp][bucket[i]];
      sh->warp_count[warp][bucket[i]] = (unsigned short)(old + __popc(same));
    }
    rank[i] = __shfl_sync(0xffffffffu, old, first) + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += blockDim.x) {          // per warp: what the warps in front of it hold
    int run = 0;
    for (int w0 = 0; w0 < n_warps; w0 += 8) {
      int c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = w0 + w < n_warps ? sh->warp_count[w0 + w][e] : 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        if (w0 + w < n_warps) sh->warp_count[w0 + w][e] = (unsigned short)run;
        run += c[w];
      }
    }
    sh->mine[e] = run;
    if (n_chunks == 1) sh->total[e] = run;
  }
  if (kCluster) {
    tc::cluster_sync_all();
    for (int e = threadIdx.x; e <= E; e += blockDim.x) {
      int other[kOrdCluster], all = 0, pre = 0;
#pragma unroll
      for (int r = 0; r < kOrdCluster; ++r) {
        other[r] = 0;
        if (r < n_chunks) asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(other[r]) : "r"(tc::mapa_cluster(tc::smem_u32(&sh->mine[e]), r)));
      }
#pragma unroll
      for (int r = 0; r < kOrdCluster; ++r) {
        all += other[r];
        pre += r < (int)blockIdx.x ? other[r] : 0;
      }
      sh->total[e] = all;
      sh->before[e] = pre;
    }
  } else if (scanned) {
    for (int e = threadIdx.x; e <= E; e += blockDim.x) {
      sh->before[e] = hist[(size_t)blockIdx.x * hist_stride(E) + e];
      sh->total[e] = hist[(size_t)n_chunks * hist_stride(E) + e];
    }
  } else if (n_chunks > 1) {                             // four columns a thread, the chunks dealt to the threads left over
    const int wide = hist_stride(E) / 4, parts = (int)blockDim.x / wide, part = threadIdx.x / wide, col = threadIdx.x % wide;
    if (part < parts) {
      const int4* rows = reinterpret_cast<const int4*>(hist) + col;
      int4 sum = make_int4(0, 0, 0, 0), pre = make_int4(0, 0, 0, 0);
#pragma unroll 8
      for (int c = part; c < n_chunks; c += parts) {
        const int4 h = rows[(size_t)c * wide];
        const int in = c < (int)blockIdx.x ? -1 : 0;
        sum.x += h.x; sum.y += h.y; sum.z += h.z; sum.w += h.w;
        pre.x += h.x & in; pre.y += h.y & in; pre.z += h.z & in; pre.w += h.w & in;
      }
      const int s4[4] = {sum.x, sum.y, sum.z, sum.w}, p4[4] = {pre.x, pre.y, pre.z, pre.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * col + i <= E) {
          atomicAdd(&sh->total[4 * col + i], s4[i]);
          atomicAdd(&sh->before[4 * col + i], p4[i]);
        }
    }
  }
  __syncthreads();
  // exclusive sums over the buckets: of the call's counts (where an expert begins in `order`) and of the chunk's (in `sorted`)
  if (warp < 2) {
    const int* from = warp == 0 ? sh->total : sh->mine;
    int run = 0;
    for (int e0 = 0; e0 <= E; e0 += 32) {
      const int e = e0 + lane, v = e <= E ? from[e] : 0;
      int inc = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (e <= E) {
        if (warp == 0) {
          sh->before[e] += run + inc - v;
          if (blockIdx.x == 0) offsets[e] = run + inc - v;      // offsets[E]: entries with an expert
        } else {
          sh->start[e] = run + inc - v;
        }
      }
      run += __shfl_sync(0xffffffffu, inc, 31);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * 32 + lane;
    if (i < steps && at < in_chunk) {
      const int e = bucket[i], in = sh->warp_count[warp][e] + rank[i];
      sh->sorted[sh->start[e] + in] = (unsigned)at | (unsigned)e << 16;
      position[chunk + at] = e < E ? sh->before[e] + in : -1;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < in_chunk; i += blockDim.x) {
    const unsigned v = sh->sorted[i];
    const int e = (int)(v >> 16);
    order[sh->before[e] + i - sh->start[e]] = e < E ? chunk + (int)(v & 0xffffu) : -1;
  }
  if (kCluster) tc::cluster_sync_all();                  // the counts stay until all have read them
}

template <typename T>
cudaError_t topk_launch(const void* logits, long long ld, int T_rows, int E, int k, int act, int renorm, const int* n_live, int* idx,
                        float* weights, cudaStream_t s) {
  const int vec = (((uintptr_t)logits | (uintptr_t)(ld * (long long)sizeof(T))) & 15u) == 0;
#define MIX_TOPK(G, V)                                                                                                          \
  return launch_pdl(kPdlHook, router_topk_kernel<T, G, V>, dim3((unsigned)(((long long)T_rows * G + kSelThreads - 1) / kSelThreads)), \
                    dim3(kSelThreads), 0, s, static_cast<const T*>(logits), ld, vec, T_rows, E, k, act, renorm, n_live, idx, weights)
  MIX_ROW_LAYOUT(E, MIX_TOPK);
#undef MIX_TOPK
}
template <typename T>
cudaError_t topk_grad_launch(const void* logits, long long ld, int T_rows, int E, int k, int act, int renorm, const int* idx,
                             const float* weights, const float* d_weights, void* d_logits, long long ld_d, cudaStream_t s) {
  const int vec = (((uintptr_t)logits | (uintptr_t)(ld * (long long)sizeof(T))) & 15u) == 0;
  const int vec_d = (((uintptr_t)d_logits | (uintptr_t)(ld_d * (long long)sizeof(T))) & 15u) == 0;
#define MIX_TOPK_GRAD(G, V)                                                                                                          \
  return launch_pdl(kPdlHook, router_topk_grad_kernel<T, G, V>, dim3((unsigned)(((long long)T_rows * G + kSelThreads - 1) / kSelThreads)), \
                    dim3(kSelThreads), 0, s, static_cast<const T*>(logits), ld, vec, T_rows, E, k, act, renorm, idx, weights, d_weights,  \
                    static_cast<T*>(d_logits), ld_d, vec_d)
  MIX_ROW_LAYOUT(E, MIX_TOPK_GRAD);
#undef MIX_TOPK_GRAD
}

}  // namespace

namespace mix {
int router_args(const void* logits, int dtype, long long ld, int T, int E, int k, int act, char* errbuf, int errbuf_len) {
  if (op_elem_size(dtype) == 0) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "dtype %d is no MIX_DTYPE_*", dtype);
  if (act != MIX_ACT_SOFTMAX && act != MIX_ACT_SIGMOID) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "act %d is neither softmax nor sigmoid", act);
  if (T < 0 || T > kOpMaxRows) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "T %d outside [0, %d]", T, kOpMaxRows);
  if (E < 1 || E > kOpMaxExperts) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n_experts %d outside [1, %d]", E, kOpMaxExperts);
  if (k < 1 || k > kOpMaxTopk || k > E) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "k %d outside [1, min(%d, n_experts)]", k, kOpMaxTopk);
  if (ld < E) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row stride %lld is below n_experts %d", ld, E);
  if (T > 0 && !logits) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "logits is NULL");
  return MIX_OK;
}
}  // namespace mix

extern "C" int mix_router_topk(const void* logits, int dtype, long long ld, int T, int n_experts, int k, int act, int renormalise,
                               const int* n_live, int* idx, float* weights, void* stream, char* errbuf, int errbuf_len) {
  const int rc = router_args(logits, dtype, ld, T, n_experts, k, act, errbuf, errbuf_len);
  if (rc != MIX_OK) return rc;
  if (T == 0) return MIX_OK;
  if (!idx || !weights) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "idx and weights are required");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == MIX_DTYPE_F32) e = topk_launch<float>(logits, ld, T, n_experts, k, act, renormalise, n_live, idx, weights, s);
  else if (dtype == MIX_DTYPE_BF16) e = topk_launch<__nv_bfloat16>(logits, ld, T, n_experts, k, act, renormalise, n_live, idx, weights, s);
  else e = topk_launch<__half>(logits, ld, T, n_experts, k, act, renormalise, n_live, idx, weights, s);
  MIX_OP_CUDA(e);
  return MIX_OK;
}

extern "C" int mix_router_topk_grad(const void* logits, int dtype, long long ld, int T, int n_experts, int k, int act, int renormalise,
                                    const int* idx, const float* weights, const float* d_weights, void* d_logits, long long ld_d,
                                    void* stream, char* errbuf, int errbuf_len) {
  const int rc = router_args(logits, dtype, ld, T, n_experts, k, act, errbuf, errbuf_len);
  if (rc != MIX_OK) return rc;
  if (ld_d < n_experts) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row stride %lld of d_logits is below n_experts %d", ld_d, n_experts);
  if (T == 0) return MIX_OK;
  if (!idx || !weights || !d_weights || !d_logits) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "idx, weights, d_weights and d_logits are required");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == MIX_DTYPE_F32) e = topk_grad_launch<float>(logits, ld, T, n_experts, k, act, renormalise, idx, weights, d_weights, d_logits, ld_d, s);
  else if (dtype == MIX_DTYPE_BF16) e = topk_grad_launch<__nv_bfloat16>(logits, ld, T, n_experts, k, act, renormalise, idx, weights, d_weights, d_logits, ld_d, s);
  else e = topk_grad_launch<__half>(logits, ld, T, n_experts, k, act, renormalise, idx, weights, d_weights, d_logits, ld_d, s);
  MIX_OP_CUDA(e);
  return MIX_OK;
}

namespace {
// How a call's entries are dealt.  What a step of a warp costs is instructions, some 90, so a chunk is small and many SMs share the
// work: 16384 entries are on 8 SMs of 512 threads, beyond that chunks of 2048.  (65536 entries of 256 experts: 9.3 us, 12.5 in eight
// chunks of 8192; 16384: 7.2, 12.3 in two; 524288: 13.3, 14.9 in 64 chunks of 8192 whose CTAs add up all chunks' counts.)
struct OrderPlan {
  int threads, steps, chunks;
  bool cluster, counts, scan;
};
OrderPlan order_plan(long long n) {
  OrderPlan p = {512, 4, 1, false, false, false};
  const auto chunks = [&](int threads, int steps) { return (int)((n + threads * steps - 1) / (threads * steps)); };
  if (n <= 512) {
    p.threads = n <= 64 ? 64 : (int)((n + 31) / 32 * 32);
    p.steps = 1;
  } else if (n <= 8 * 2048) {                                  // one cluster, 512 entries or more a CTA
    p.chunks = n <= 1024 ? 2 : (n <= 2048 ? 4 : kOrdCluster);
    p.threads = n <= 4096 ? 256 : 512;
    p.steps = (int)((n + (long long)p.threads * p.chunks - 1) / ((long long)p.threads * p.chunks));
    p.chunks = chunks(p.threads, p.steps);
    p.cluster = p.chunks > 1;
  } else {
    p.chunks = chunks(p.threads, p.steps);
    p.scan = p.chunks > 64;
    p.counts = true;
  }
  return p;
}
}  // namespace

extern "C" long long mix_expert_order_workspace(long long n, int n_experts) {
  if (n < 0 || n > MIX_ORDER_MAX_ENTRIES || n_experts < 1 || n_experts > kOpMaxExperts) return MIX_ERR_OUT_OF_RANGE;
  const OrderPlan p = order_plan(n);
  return p.counts ? (long long)(p.chunks + 1) * hist_stride(n_experts) * (long long)sizeof(int) : 0;
}

extern "C" int mix_expert_order(const int* idx, long long n, int n_experts, int* offsets, int* order, int* position, void* workspace,
                                long long workspace_bytes, void* stream, char* errbuf, int errbuf_len) {
  if (n_experts < 1 || n_experts > kOpMaxExperts) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n_experts %d outside [1, %d]", n_experts, kOpMaxExperts);
  if (n < 0 || n > MIX_ORDER_MAX_ENTRIES) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n %lld outside [0, %d]", n, MIX_ORDER_MAX_ENTRIES);
  if (!offsets || (n > 0 && (!idx || !order || !position))) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "idx, offsets, order and position are required");
  const long long need = mix_expert_order_workspace(n, n_experts);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15u)))
    MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "the workspace has to hold %lld bytes, on 16 bytes", need);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int* hist = static_cast<int*>(workspace);
  const OrderPlan p = order_plan(n);
  static std::atomic<int> ready[kOpDevices];
  int dev, n_sms;
  MIX_OP_CUDA(op_device(&dev, &n_sms));
  if (!ready[dev].load(std::memory_order_relaxed)) {
    MIX_OP_CUDA(cudaFuncSetAttribute(expert_order_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(OrderShared)));
    MIX_OP_CUDA(cudaFuncSetAttribute(expert_order_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(OrderShared)));
    ready[dev].store(1, std::memory_order_relaxed);
  }
  if (p.counts) MIX_OP_CUDA(launch_pdl(kPdlHook, expert_hist_kernel, dim3(p.chunks), dim3(p.threads), 0, s, idx, (int)n, n_experts, p.steps, hist));
  if (p.scan) MIX_OP_CUDA(launch_pdl(kPdlHook, expert_scan_kernel, dim3((hist_stride(n_experts) + 31) / 32), dim3(kScanThreads), 0, s, hist, p.chunks, hist_stride(n_experts)));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.chunks);
  cfg.blockDim = dim3(p.threads);
  cfg.dynamicSmemBytes = sizeof(OrderShared);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  int n_at = 0;
  if (p.cluster) {
    at[n_at].id = cudaLaunchAttributeClusterDimension;
    at[n_at].val.clusterDim.x = p.chunks;
    at[n_at].val.clusterDim.y = 1;
    at[n_at++].val.clusterDim.z = 1;
  }
  if (pdl_mask() & kPdlHook) {
    at[n_at].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n_at++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = at;
  cfg.numAttrs = n_at;
  MIX_OP_CUDA(cudaLaunchKernelEx(&cfg, p.cluster ? expert_order_kernel<true> : expert_order_kernel<false>, idx, (int)n, n_experts,
                                 static_cast<const int*>(hist), p.chunks, p.steps, (int)p.scan, offsets, order, position));
  return MIX_OK;
}

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

using namespace mix;

namespace {

constexpr int kSelThreads = 256;

// ---------------------------------------------------------------------------------------------------- selection
// The selection compares the logits themselves, never probabilities: those round, and two logits that differ could tie.
//
// Rows of up to 128 experts: k rounds of an arg-max over the G lanes, 32 / G rows of a warp side by side.
// Wider rows (a warp each): the k-th largest of the lanes' own largest logits is a lower bound on the row's k-th largest logit,
// and only a few more than k logits reach it.  Those go to shared memory, one to a lane, and each counts how many come before it.
// Where more than 32 reach it (many equal logits) the rounds decide.  65536 rows of 256, k = 8, with the softmax over the row:
// 76 us by rounds, %s us so; the logits' stream alone takes 10.3.
constexpr int kSelWarps = kSelThreads / 32;
template <typename T, int G, int V>
__global__ void __launch_bounds__(kSelThreads)
router_topk_kernel(const T* __restrict__ logits, long long ld, int vec, int T_rows, int E, int k, int act, int renorm,
                   const int* __restrict__ n_live, int* __restrict__ idx, float* __restrict__ weights) {
  constexpr int S = G >= kOpMaxTopk ? 1 : (G == 1 ? 8 : kOpMaxTopk / G);   // chosen entries a lane keeps: entry j is lane j % G's
  __shared__ float2 found[G == 32 ? kSelWarps : 1][32];                    // (logit, column)
  pdl_wait();
  pdl_launch_dependents();
  const int sub = threadIdx.x & (G - 1);
  const long long t = ((long long)blockIdx.x * kSelThreads + threadIdx.x) / G;
  const int live = n_live ? min(*n_live, T_rows) : T_rows;
  float x[V];
  if (t < live) {
    load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = -INFINITY;
  }
  const float lane_top = top_of<V>(x), top = group_max<G>(lane_top);
  int my_idx[S];
  float my_x[S];
#pragma unroll
  for (int s = 0; s < S; ++s) { my_idx[s] = -1; my_x[s] = -INFINITY; }
  bool rounds = true;
  if (G == 32) {
    const int warp = threadIdx.x >> 5;
    float rest = lane_top, bound = -INFINITY;
    for (int left = k; left > 0;) {
      bound = group_max<32>(rest);
      if (bound == -INFINITY) break;
      const unsigned at = __ballot_sync(0xffffffffu, rest == bound);
      left -= __popc(at);
      if (rest == bound) rest = -INFINITY;
    }
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool in = x[v] >= bound && x[v] > -INFINITY;
      const unsigned at = __ballot_sync(0xffffffffu, in);
      const int to = n + __popc(at & ((1u << sub) - 1u));
      if (in && to < 32) found[warp][to] = make_float2(x[v], __int_as_float(row_col<T, G>(v, sub)));
      n += __popc(at);
    }
    if (n <= 32) {
      rounds = false;
      __syncwarp();
      const float2 mine = found[warp][sub];
      const int col = __float_as_int(mine.y);
      int rank = 0;
      for (int i = 0; i < n; ++i) {
        const float2 f = found[warp][i];
        rank += f.x > mine.x || (f.x == mine.x && __float_as_int(f.y) < col);
      }
      __syncwarp();
      if (sub < n) found[warp][rank] = mine;                               // in the order of the ranks
      __syncwarp();
      if (sub < n && sub < k) {
        my_x[0] = found[warp][sub].x;
        my_idx[0] = __float_as_int(found[warp][sub].y);
      }
    }
  }
  if (rounds) {
    float key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = x[v];
#pragma unroll
    for (int j = 0; j < (G == 1 ? 8 : kOpMaxTopk); ++j) {
      if (j >= k) break;
      const float m = group_max<G>(top_of<V>(key));
      unsigned c = 0xffffffffu;
#pragma unroll
      for (int v = V - 1; v >= 0; --v) c = key[v] == m ? (unsigned)row_col<T, G>(v, sub) : c;   // (columns rise with v)
      if (G == 32) {
        c = __reduce_min_sync(0xffffffffu, c);
      } else {
#pragma unroll
        for (int o = 1; o < G; o <<= 1) c = min(c, __shfl_xor_sync(0xffffffffu, c, o));
      }
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = (unsigned)row_col<T, G>(v, sub) == c ? -INFINITY : key[v];
      if (j % G == sub && m > -INFINITY) {
        my_idx[j / G] = (int)c;
        my_x[j / G] = m;
      }
    }
  }
  const bool plain = act == MIX_ACT_SIGMOID && !renorm;                    // the weight is the sigmoid itself
  float total = 0.f;
  if (act == MIX_ACT_SOFTMAX && !renorm) total = scores<V>(act, top, x);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    my_x[s] = my_idx[s] < 0 ? 0.f : (plain ? sigmoid_row(my_x[s]) : score(act, my_x[s], top));
    if (renorm) total += my_x[s];
  }
  if (!plain) total = group_sum<G>(total);
  if (t >= T_rows) return;
  const float norm = plain ? 1.f : total;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int j = s * G + sub;
    if (j < k) {
      idx[t * k + j] = my_idx[s];
      weights[t * k + j] = my_idx[s] >= 0 ? my_x[s] / norm : 0.f;
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
// The chosen entries are spread over the row through shared memory where a lane has one of them (more than 64 experts): each lane
// puts its own where its column is, and the row comes back in the lanes' pieces.  Narrower rows compare each entry with each
// column of a lane, for 32 / G rows at a time.
template <typename T, int G, int V>
__global__ void __launch_bounds__(kSelThreads)
router_topk_grad_kernel(const T* __restrict__ logits, long long ld, int vec, int T_rows, int E, int k, int act, int renorm,
                        const int* __restrict__ idx, const float* __restrict__ weights, const float* __restrict__ d_weights,
                        T* __restrict__ d_logits, long long ld_d, int vec_d) {
  constexpr int S = G >= kOpMaxTopk ? 1 : (G == 1 ? 8 : kOpMaxTopk / G);
  __shared__ float4 spread[S == 1 ? kSelThreads * V / 4 : 1];
  pdl_wait();
  pdl_launch_dependents();
  const int sub = threadIdx.x & (G - 1);
  const long long t = ((long long)blockIdx.x * kSelThreads + threadIdx.x) / G;
  const bool row = t < T_rows, dense = act == MIX_ACT_SOFTMAX && !renorm;
  float d[V], p[V];
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = -INFINITY;
  if (dense && row) load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, p);
  int my_idx[S];
  float my_g[S], my_w[S];
  float s = 0.f;
  bool any = false;
#pragma unroll
  for (int i = 0; i < S; ++i) {
    const int j = i * G + sub;
    my_idx[i] = row && j < k ? idx[t * k + j] : -1;
    const bool ok = (unsigned)my_idx[i] < (unsigned)E;
    if (!ok) my_idx[i] = -1;
    my_g[i] = ok ? d_weights[t * k + j] : 0.f;
    my_w[i] = ok ? weights[t * k + j] : 0.f;
    s += my_g[i] * my_w[i];
    any |= ok;
  }
  s = group_sum<G>(s);
  if (dense) {
    any = group_any<G>(any);
    const float total = group_sum<G>(scores<V>(act, group_max<G>(top_of<V>(p)), p));
    const float inv = any && total > 0.f ? 1.f / total : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] *= inv;
  } else {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      float g = my_w[i] * ((act == MIX_ACT_SOFTMAX || renorm) ? my_g[i] - s : my_g[i]);
      if (act == MIX_ACT_SIGMOID && my_idx[i] >= 0) g *= sigmoid_row(-to_f32(logits[t * ld + my_idx[i]]));
      my_g[i] = my_idx[i] >= 0 ? g : 0.f;
    }
  }
  if (S == 1) {
    constexpr int VW = RowVec<T>::VW;
    const int lane = threadIdx.x & 31;
    float* buf = reinterpret_cast<float*>(spread) + (threadIdx.x / G) * (G * V);
    // lane `sub`'s piece b of the row begins at column b * G * VW + sub * VW
#pragma unroll
    for (int b = 0; b < V / 4; ++b)
      *reinterpret_cast<float4*>(buf + (b * 4 / VW) * (G * VW) + sub * VW + (b * 4) % VW) = make_float4(0.f, 0.f, 0.f, 0.f);
    // the same expert twice in a row (never in what the selection gives): its entries are added in their order
    const unsigned same = __match_any_sync(0xffffffffu, my_idx[0] < 0 ? -1 - lane : my_idx[0] + (lane / G) * kOpMaxExperts);
    float g = my_g[0];
    if (__any_sync(0xffffffffu, (same & (same - 1u)) != 0u)) {
      g = 0.f;
      for (int i = 0; i < 32; ++i) {
        const float x = __shfl_sync(0xffffffffu, my_g[0], i);
        if ((same >> i) & 1u) g += x;
      }
    }
    __syncwarp();
    if (my_idx[0] >= 0 && lane == __ffs(same) - 1) buf[my_idx[0]] = g;
    __syncwarp();
#pragma unroll
    for (int b = 0; b < V / 4; ++b) {
      const float4 f = *reinterpret_cast<const float4*>(buf + (b * 4 / VW) * (G * VW) + sub * VW + (b * 4) % VW);
      d[4 * b] = f.x;
      d[4 * b + 1] = f.y;
      d[4 * b + 2] = f.z;
      d[4 * b + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = 0.f;
#pragma unroll
    for (int j = 0; j < (G == 1 ? 8 : kOpMaxTopk); ++j) {
      if (j >= k) break;
      const int at = __shfl_sync(0xffffffffu, my_idx[j / G], j % G, G);
      const float g = __shfl_sync(0xffffffffu, my_g[j / G], j % G, G);
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] += row_col<T, G>(v, sub) == at ? g : 0.f;
    }
  }
  if (dense) {
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = p[v] > 0.f ? p[v] * (d[v] - s) : 0.f;
  }
  if (row) store_row<T, G, V>(d_logits + t * ld_d, E, sub, vec_d != 0, d);
}

// ---------------------------------------------------------------------------------------------------- order by expert
constexpr int kOrdThreads = 512;
constexpr int kOrdWarps = kOrdThreads / 32;
constexpr int kOrdSteps = 8;                                    // entries a lane takes
constexpr int kOrdChunk = kOrdThreads * kOrdSteps;              // entries a CTA takes
constexpr int kOrdBuckets = kOpMaxExperts + 1;                  // the last of a call's holds the entries without an expert

__host__ __device__ constexpr int hist_stride(int E) { return (E + 1 + 3) & ~3; }   // counts of a chunk, in whole 16-byte vectors
__device__ __forceinline__ int bucket_of(int i, int E) { return (unsigned)i < (unsigned)E ? i : E; }

__global__ void __launch_bounds__(kOrdThreads)
expert_hist_kernel(const int* __restrict__ idx, int n, int E, int* __restrict__ hist) {
  __shared__ int h[kOrdBuckets];
  pdl_wait();
  pdl_launch_dependents();
  for (int e = threadIdx.x; e <= E; e += kOrdThreads) h[e] = 0;
  __syncthreads();
  const int base = blockIdx.x * kOrdChunk;
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * kOrdThreads + threadIdx.x;
    if (at < n) atomicAdd(&h[bucket_of(idx[at], E)], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < hist_stride(E); e += kOrdThreads) hist[(size_t)blockIdx.x * hist_stride(E) + e] = e <= E ? h[e] : 0;
}

// Entry i of the CTA's chunk goes to  (entries of lower experts) + (entries of this expert in earlier chunks, in earlier warps
// of the CTA, earlier in the warp).  The counts of the other chunks come from expert_hist_kernel; one chunk needs none, and a
// call of up to 4096 entries is this one launch.
__global__ void __launch_bounds__(kOrdThreads)
expert_order_kernel(const int* __restrict__ idx, int n, int E, const int* __restrict__ hist, int n_chunks, int* __restrict__ offsets,
                    int* __restrict__ order, int* __restrict__ position) {
  __shared__ int warp_count[kOrdWarps][kOrdBuckets];
  __shared__ int total[kOrdBuckets], before[kOrdBuckets];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int e = threadIdx.x; e <= E; e += kOrdThreads) {
    total[e] = 0;
    before[e] = 0;
    for (int w = 0; w < kOrdWarps; ++w) warp_count[w][e] = 0;
  }
  __syncthreads();
  const int base = blockIdx.x * kOrdChunk + warp * (32 * kOrdSteps);
  int bucket[kOrdSteps], rank[kOrdSteps];
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * 32 + lane;
    bucket[i] = at < n ? bucket_of(idx[at], E) : kOrdBuckets;
  }
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const unsigned same = __match_any_sync(0xffffffffu, bucket[i]);
    const int first = __ffs(same) - 1;
    int old = 0;
    if (lane == first && bucket[i] < kOrdBuckets) {
      old = warp_count[warp][bucket[i]];
      warp_count[warp][bucket[i]] = old + __popc(same);
    }
    rank[i] = __shfl_sync(0xffffffffu, old, first) + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
  }
  __syncthreads();
  if (n_chunks > 1) {                                    // four columns a thread, the chunks dealt to the threads left over
    const int wide = hist_stride(E) / 4, parts = kOrdThreads / wide, part = threadIdx.x / wide, col = threadIdx.x % wide;
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
          atomicAdd(&total[4 * col + i], s4[i]);
          atomicAdd(&before[4 * col + i], p4[i]);
        }
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += kOrdThreads) {   // per warp: what the warps in front of it hold
    int run = before[e];
#pragma unroll
    for (int w = 0; w < kOrdWarps; ++w) {
      const int c = warp_count[w][e];
      warp_count[w][e] = run;
      run += c;
    }
    if (n_chunks == 1) total[e] = run;
  }
  __syncthreads();
  if (warp == 0) {                                       // exclusive sum over the buckets
    constexpr int kEach = (kOrdBuckets + 31) / 32;
    int v[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = lane * kEach + i;
      v[i] = e <= E ? total[e] : 0;
      sum += v[i];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    int run = inc - sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = lane * kEach + i;
      if (e <= E) {
        total[e] = run;
        if (blockIdx.x == 0) offsets[e] = run;           // offsets[E]: entries with an expert
      }
      run += v[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOrdSteps; ++i) {
    const int at = base + i * 32 + lane;
    if (at < n) {
      const int b = bucket[i], to = total[b] + warp_count[warp][b] + rank[i];
      order[to] = b < E ? at : -1;
      position[at] = b < E ? to : -1;
    }
  }
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
  if (T < 0) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "T %d is negative", T);
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

extern "C" long long mix_expert_order_workspace(long long n, int n_experts) {
  if (n < 0 || n > MIX_ORDER_MAX_ENTRIES || n_experts < 1 || n_experts > kOpMaxExperts) return MIX_ERR_OUT_OF_RANGE;
  const long long chunks = (n + kOrdChunk - 1) / kOrdChunk;
  return chunks > 1 ? chunks * hist_stride(n_experts) * (long long)sizeof(int) : 0;
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
  const int chunks = n == 0 ? 1 : (int)((n + kOrdChunk - 1) / kOrdChunk);
  if (chunks > 1) MIX_OP_CUDA(launch_pdl(kPdlHook, expert_hist_kernel, dim3(chunks), dim3(kOrdThreads), 0, s, idx, (int)n, n_experts, hist));
  MIX_OP_CUDA(launch_pdl(kPdlHook, expert_order_kernel, dim3(chunks), dim3(kOrdThreads), 0, s, idx, (int)n, n_experts, static_cast<const int*>(hist),
                         chunks, offsets, order, position));
  return MIX_OK;
}

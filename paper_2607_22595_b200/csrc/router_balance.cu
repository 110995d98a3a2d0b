// How evenly a router spreads the tokens of each request over its experts, and the loss on it.
//
// For a segment s of rows (a request), n_s of which name an expert, with C_e = how often they name expert e:
//   f_e = C_e / sum C        P_e = mean over the n_s rows of p_te        L_s = E sum_e f_e P_e
//   dL_s / dx_tj = E / n_s  p_tj (f_j - sum_e f_e p_te)  [(1 - sigmoid(x_tj))  where the scores are sigmoids]
// f counts, so no gradient passes through it.
//
// Forward: one pass over the logits.  A CTA (unit u) takes a run of rows, walks the segments that the run touches and leaves
// what it saw of each in slot u + s of the partial sums -- along the runs and segments either u or s goes up by one at every
// step, so no two share a slot, and which row is added where never depends on timing.  A second launch adds the slots up, a
// cluster of CTAs per segment where a segment has many.  Both add in a fixed order.
// Backward: one pass over the logits, a warp per run of rows.
//
// 65536 rows of 256 fp32 in 16 segments, k = 8, sigmoid: forward 28.0 us (21 and 7 in its two launches; the logits' stream takes 10.3),
// backward 29.8 (20.6 read and written).  What bounds both is issue: 14 instructions a logit, two of them on the special-function
// unit, beside the reductions of a row.
#include "op_common.cuh"
#include "tc_common.cuh"

using namespace mix;

namespace {

constexpr int kUnitWarps = 8;              // warps of a unit where requests are long
// CTAs an SM holds at a time: large batches make whole waves of them.  Above 256 experts, with 16 logits a lane, the backward spills 140 bytes
// for it (the forward of small calls 32, the forward in units nothing) and is faster all the same: 32768 rows of 512 fp32, forward 23.9
// us and backward 31.3, 27.1 and 32.7 with three and two CTAs.
constexpr int kUnitCtas = 4, kGradCtas = 4;
constexpr int kFinThreads = 512;
constexpr int kFinCluster = 8;

// Offset i of n_seg segments, in [0, T] whatever stands in the table; without a table all rows are one segment.
__device__ __forceinline__ int seg_at(const int* __restrict__ seg, int i, int T) { return seg ? min(max(seg[i], 0), T) : (i == 0 ? 0 : T); }

// The last segment that begins at or before row r (0 where none does), found by a whole warp: 32 probes a step.
__device__ __forceinline__ int seg_of_row(const int* __restrict__ seg, int n_seg, int T, int r, int lane) {
  int lo = 0, n = n_seg;                                       // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const unsigned ok = __ballot_sync(0xffffffffu, lane * step < n && seg_at(seg, at, T) <= r);
    const int i = ok ? 31 - __clz(ok) : 0;
    n = min(step, n - i * step);
    lo += i * step;
  }
  return lo;
}

// direct: unit u IS segment u, and the CTA that has seen all of it writes its results itself.
struct BalanceOut {
  float* loss;
  int* counts;
  float* mean_p;
  int* rows;
};
template <typename T, int G, int V, int W, bool kDirect>
__global__ void __launch_bounds__(32 * W, W == kUnitWarps ? kUnitCtas : 1)
balance_kernel(const T* __restrict__ logits, long long ld, int vec, const int* __restrict__ idx, int T_rows, int E, int k, int act,
               const int* __restrict__ seg, int n_seg, int unit_rows, float* __restrict__ part_p, int* __restrict__ part_c,
               int* __restrict__ part_n, const BalanceOut out) {
  constexpr int R = 32 / G;                                    // rows a warp holds
  __shared__ double red[W];
  __shared__ long long red_c[W];
  __shared__ int hist[G * V];
  __shared__ float sum_p[W][G * V];
  __shared__ int sum_n[W];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (G - 1), unit = blockIdx.x;
  const int r0 = kDirect ? seg_at(seg, unit, T_rows) : unit * unit_rows, r1 = kDirect ? seg_at(seg, unit + 1, T_rows) : min(T_rows, r0 + unit_rows);
  for (int e = threadIdx.x; e < G * V; e += 32 * W) hist[e] = 0;
  if (W > 1) __syncthreads(); else __syncwarp();
  for (int s = kDirect ? unit : seg_of_row(seg, n_seg, T_rows, r0, lane); s < (kDirect ? unit + 1 : n_seg); ++s) {
    const int a = kDirect ? r0 : max(seg_at(seg, s, T_rows), r0), b = kDirect ? r1 : min(seg_at(seg, s + 1, T_rows), r1);
    if (!kDirect && a >= r1) break;
    if (!kDirect && a >= b) continue;
    float acc[V];
    int rows = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.f;
    // The next row is under way while one is worked on: a warp has few rows, and a row's reductions are one after the other.
    const auto fetch = [&](int base, float (&x)[V], int& name) {
      const int t = base + lane / G;
      name = -1;
      if (t < b) {
        load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
        if (sub < k) name = idx[(long long)t * k + sub];
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = -INFINITY;
      }
    };
    float next[V];
    int next_name;
    fetch(a + warp * R, next, next_name);
    for (int base = a + warp * R; base < b; base += W * R) {   // (all lanes of a warp: a row of no segment is a row that is off)
      const int t = base + lane / G;
      float x[V];
      const int name = next_name;
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = next[v];
      fetch(base + W * R, next, next_name);
      bool named = (unsigned)name < (unsigned)E;
      if (named) atomicAdd(&hist[name], 1);
      if (G < kOpMaxTopk && t < b) {                           // (a lane's further entries of a narrow row)
        for (int j = sub + G; j < k; j += G) {
          const int i = idx[(long long)t * k + j];
          if ((unsigned)i < (unsigned)E) {
            atomicAdd(&hist[i], 1);
            named = true;
          }
        }
      }
      const bool on = group_any<G>(named);
      rows += on && sub == 0;
      float total = group_sum<G>(scores<V>(act, act == MIX_ACT_SOFTMAX ? group_max<G>(top_of<V>(x)) : 0.f, false, x));
      if (act == MIX_ACT_SIGMOID && __any_sync(0xffffffffu, on && total < kLowTotal)) {
        if (t < b) load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
        total = group_sum<G>(scores<V>(act, group_max<G>(top_of<V>(x)), true, x));
      }
      const float inv = on && total > 0.f ? rcp_hw(total) : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] = fmaf(x[v], inv, acc[v]);
    }
    // this segment's share of the unit
#pragma unroll
    for (int o = G; o < 32; o <<= 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] += __shfl_xor_sync(0xffffffffu, acc[v], o);
    }
    rows = __reduce_add_sync(0xffffffffu, rows);
    if (lane < G) {
#pragma unroll
      for (int v = 0; v < V; ++v) sum_p[warp][row_col<T, G>(v, sub)] = acc[v];
    }
    if (lane == 0) sum_n[warp] = rows;
    if (W > 1) __syncthreads(); else __syncwarp();
    if (kDirect) {
      int n = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) n += sum_n[w];
      double fp = 0.0;
      long long total = 0;
      for (int e = threadIdx.x; e < E; e += 32 * W) {
        double p = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) p += (double)sum_p[w][e];
        p = n > 0 ? p / n : 0.0;
        const int c = hist[e];
        out.counts[(size_t)s * E + e] = c;
        out.mean_p[(size_t)s * E + e] = (float)p;
        fp += p * c;
        total += c;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        fp += __shfl_xor_sync(0xffffffffu, fp, o);
        total += __shfl_xor_sync(0xffffffffu, total, o);
      }
      if (lane == 0) {
        red[warp] = fp;
        red_c[warp] = total;
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        for (int w = 1; w < W; ++w) {
          fp += red[w];
          total += red_c[w];
        }
        out.loss[s] = total > 0 ? (float)(E * fp / (double)total) : 0.f;
        out.rows[s] = n;
      }
      return;
    }
    const size_t slot = (size_t)(unit + s);
    for (int e = threadIdx.x; e < E; e += 32 * W) {
      float p = sum_p[0][e];
#pragma unroll
      for (int w = 1; w < W; ++w) p += sum_p[w][e];
      part_p[slot * E + e] = p;
      part_c[slot * E + e] = hist[e];
      hist[e] = 0;
    }
    if (threadIdx.x == 0) {
      int n = sum_n[0];
#pragma unroll
      for (int w = 1; w < W; ++w) n += sum_n[w];
      part_n[slot] = n;
    }
    if (W > 1) __syncthreads(); else __syncwarp();
  }
}

// One segment per cluster: CTA r of the cluster adds up the r-th part of the segment's slots, CTA 0 puts the parts together.
// Sums in 64 bits: there are few, and a long request has thousands of slots.
// (as many threads as experts where requests are short: there are many such CTAs)
template <int cluster, bool kShort>
__global__ void __launch_bounds__(kFinThreads)
balance_finish_kernel(const float* __restrict__ part_p, const int* __restrict__ part_c, const int* __restrict__ part_n, int T_rows, int E,
                      const int* __restrict__ seg, int unit_rows, float* __restrict__ loss, int* __restrict__ counts,
                      float* __restrict__ mean_p, int* __restrict__ rows_out) {
  __shared__ double sp[kOpMaxExperts];
  __shared__ int sc[kOpMaxExperts];
  __shared__ double red[kFinThreads / 32];
  __shared__ long long red_c[kFinThreads / 32];
  __shared__ int sn;
  __shared__ double lane_p[kFinThreads];
  __shared__ int lane_c[kFinThreads];
  pdl_wait();
  pdl_launch_dependents();
  const int s = blockIdx.x / cluster, rank = blockIdx.x % cluster, tid = threadIdx.x;
  const int threads = kShort ? (int)blockDim.x : kFinThreads;
  const int a = seg_at(seg, s, T_rows), b = seg_at(seg, s + 1, T_rows);
  int u0 = 0, u1 = 0;                                          // units that the segment touches
  if (a < b) {
    u0 = a / unit_rows;
    u1 = (b - 1) / unit_rows + 1;
  }
  const int each = (u1 - u0 + cluster - 1) / cluster;
  const int v0 = min(u1, u0 + rank * each), v1 = min(u1, v0 + each);
  if (tid == 0) sn = 0;
  __syncthreads();
  {
    int n = 0;
    for (int u = v0 + tid; u < v1; u += threads) n += part_n[u + s];
    n = __reduce_add_sync(0xffffffffu, n);
    if ((tid & 31) == 0 && n) atomicAdd(&sn, n);
  }
  const int wide = (E + 31) & ~31, lanes = threads / wide;     // (threads >= wide: one pass)
  const int e = tid % wide, part = tid / wide;
  double p = 0.0;
  int c = 0;
  if (part < lanes && e < E) {
#pragma unroll 4
    for (int u = v0 + part; u < v1; u += lanes) {
      p += (double)part_p[(size_t)(u + s) * E + e];
      c += part_c[(size_t)(u + s) * E + e];
    }
  }
  lane_p[tid] = p;
  lane_c[tid] = c;
  __syncthreads();
  if (tid < wide && e < E) {
    for (int i = 1; i < lanes; ++i) {
      p += lane_p[i * wide + tid];
      c += lane_c[i * wide + tid];
    }
    sp[e] = p;
    sc[e] = c;
  }
  if (cluster > 1) tc::cluster_sync_all(); else __syncthreads();
  if (rank == 0) {
    int others[cluster];                                       // (all on their way before one is used)
#pragma unroll
    for (int r = 1; r < cluster; ++r)
      asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(others[r]) : "r"(tc::mapa_cluster(tc::smem_u32(&sn), r)));
    int n = sn;
    double fp = 0.0;
    long long total = 0;
    if (tid < E) {
      double op[cluster];
      int oc[cluster];
#pragma unroll
      for (int r = 1; r < cluster; ++r) {
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(op[r]) : "r"(tc::mapa_cluster(tc::smem_u32(&sp[tid]), r)));
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(oc[r]) : "r"(tc::mapa_cluster(tc::smem_u32(&sc[tid]), r)));
      }
      p = sp[tid];
      c = sc[tid];
#pragma unroll
      for (int r = 1; r < cluster; ++r) {
        p += op[r];
        c += oc[r];
      }
    }
#pragma unroll
    for (int r = 1; r < cluster; ++r) n += others[r];
    if (tid < E) {
      p = n > 0 ? p / n : 0.0;
      counts[(size_t)s * E + tid] = c;
      mean_p[(size_t)s * E + tid] = (float)p;
      fp = p * c;
      total = c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      fp += __shfl_xor_sync(0xffffffffu, fp, o);
      total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if ((tid & 31) == 0) {
      red[tid >> 5] = fp;
      red_c[tid >> 5] = total;
    }
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < threads / 32; ++w) {
        fp += red[w];
        total += red_c[w];
      }
      loss[s] = total > 0 ? (float)(E * fp / (double)total) : 0.f;
      rows_out[s] = n;
    }
  }
  if (cluster > 1) tc::cluster_sync_all();                     // the parts stay until they have been read
}

template <typename T, int G, int V>
__global__ void __launch_bounds__(256, kGradCtas)
balance_grad_kernel(const T* __restrict__ logits, long long ld, int vec, const int* __restrict__ idx, int T_rows, int E, int k, int act,
                    const int* __restrict__ seg, int n_seg, const int* __restrict__ counts, const int* __restrict__ rows,
                    const float* __restrict__ d_loss, int warp_rows, T* __restrict__ d_logits, long long ld_d, int vec_d) {
  constexpr int R = 32 / G;
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (G - 1);
  const long long run = ((long long)blockIdx.x * 8 + warp) * warp_rows;
  if (run >= T_rows) return;                                   // (whole warps)
  const int r0 = (int)run, r1 = (int)min((long long)T_rows, run + warp_rows);
  const int s_first = seg_of_row(seg, n_seg, T_rows, r0, lane);
  int at = r0;                                                 // rows in front of `at` are done
  for (int s = s_first; at < r1; ++s) {
    // rows [at, b) belong to segment s; what no segment covers, in front of the first or behind the last, gets zeros
    const bool behind = s >= n_seg;
    const int a = behind ? r1 : min(max(seg_at(seg, s, T_rows), at), r1);
    const int b = behind ? r1 : min(max(seg_at(seg, s + 1, T_rows), a), r1);
    float f[V];
    float coef = 0.f;
    if (a < b) {
      long long total = 0;
      int c[V], most = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = row_col<T, G>(v, sub);
        c[v] = col < E ? counts[(size_t)s * E + col] : 0;
        total += c[v];
        most = max(most, c[v]);
      }
#pragma unroll
      for (int o = 1; o < G; o <<= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
      }
      // Where the experts are chosen nearly alike the largest share is taken off all of them, in whole numbers -- f_j - sum f p is the
      // same, p adds up to 1 -- so that small differences are not those of large terms (and nothing is left where all are alike).
      // Where few are chosen the shares stay: most of them are 0.
      const int off = 2 * total > (long long)E * most ? most : 0;
#pragma unroll
      for (int v = 0; v < V; ++v) f[v] = (float)(c[v] - off);
      const int n = rows[s];
      coef = n > 0 ? d_loss[s] * (float)E / (float)n : 0.f;
      const float inv = total > 0 ? 1.f / (float)total : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) f[v] *= inv;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) f[v] = 0.f;
    }
    const auto fetch = [&](int base, float (&x)[V], bool& named) {
      const int t = base + lane / G;
      named = false;
      if (t >= a && t < b) {
        load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
        for (int j = sub; j < k; j += G) named |= (unsigned)idx[(long long)t * k + j] < (unsigned)E;
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = -INFINITY;
      }
    };
    float next[V];
    bool next_named;
    fetch(at, next, next_named);
    for (int base = at; base < b; base += R) {
      const int t = base + lane / G;
      float x[V], slope[V];
      const bool on = group_any<G>(next_named);
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = next[v];
      if (base + R < b) fetch(base + R, next, next_named);
      float total = group_sum<G>(scores<V>(act, act == MIX_ACT_SOFTMAX ? group_max<G>(top_of<V>(x)) : 0.f, false, x, &slope));
      if (act == MIX_ACT_SIGMOID && __any_sync(0xffffffffu, on && total < kLowTotal)) {
        if (t >= a && t < b) load_row<T, G, V>(logits + t * ld, E, sub, vec != 0, x);
        total = group_sum<G>(scores<V>(act, group_max<G>(top_of<V>(x)), true, x, &slope));
      }
      const float inv = on && total > 0.f ? rcp_hw(total) : 0.f;
      float dot = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) dot = fmaf(f[v], x[v], dot);
      dot = group_sum<G>(dot) * inv;
      const float by = inv != 0.f ? coef * inv : 0.f;          // (a row that is off stays 0, whatever its d_loss)
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = by * slope[v] * (f[v] - dot);
      if (t < b) store_row<T, G, V>(d_logits + t * ld_d, E, sub, vec_d != 0, x);
    }
    at = b;
  }
}

struct Plan {
  int warps, unit_rows, units, cluster, direct;
  long long slots;
};
// Small calls (up to 16384 logits): a CTA per segment, one launch, which even one segment of all rows finishes in a few trips.
// Otherwise units of eight warps where the average request has 64 rows or more: one wave of CTAs, of at least 32 rows (64 requests in
// 8192 rows of 64 bf16: 9.8 us, 11.3 with 64 rows).  Where requests are short (decode steps: one row each) a unit is one warp and no
// barrier stands between two requests; each costs it a microsecond and a half, so a unit has 4 rows as long as the SMs hold all
// units at once (1024 requests of one row, 64 experts: 10.6 us, 46 with 32 rows).
// A lane adds the probabilities of an expert up in fp32, so it takes no more than 64 rows: beyond 303104 rows of more than 128 experts the
// units make several waves.  (A small call is within it: 16384 logits are 64 rows a lane at most.)
constexpr int kDirectLogits = 16384;
constexpr int kLaneRows = 64;
int rows_of_a_warp(int E) {                                     // held at a time: 32 / G of MIX_ROW_LAYOUT
  int rows = 32;
  while (rows > 1 && 256 / rows < E) rows /= 2;
  return rows;
}
Plan plan(int T, int E, int n_seg, int n_sms) {
  Plan p;
  p.direct = (long long)T * E <= kDirectLogits;
  p.warps = T / n_seg >= 64 ? kUnitWarps : 1;
  if (p.warps == kUnitWarps) {
    const int wave = kUnitCtas * n_sms, most = kUnitWarps * rows_of_a_warp(E) * kLaneRows, waves = (T - 1) / (wave * most) + 1;
    p.unit_rows = (T - 1) / (wave * waves) + 1;
    if (p.unit_rows < 32) p.unit_rows = 32;
  } else {
    p.unit_rows = T <= 8 * 32 * n_sms ? 4 : 32;
  }
  p.units = T > 0 ? (T + p.unit_rows - 1) / p.unit_rows : 0;
  p.slots = p.direct ? 0 : (long long)p.units + n_seg;
  p.cluster = p.units / n_seg >= 16 ? kFinCluster : 1;
  return p;
}
long long workspace_bytes_of(const Plan& p, int E) { return p.slots * (8ll * E + 4); }

template <typename T, int G, int V, int W, bool kDirect>
cudaError_t balance_launch_one(const Plan& p, const void* logits, long long ld, const int* idx, int T_rows, int E, int k, int act, const int* seg,
                               int n_seg, float* part_p, int* part_c, int* part_n, const BalanceOut& out, cudaStream_t s) {
  const int vec = (((uintptr_t)logits | (uintptr_t)(ld * (long long)sizeof(T))) & 15u) == 0;
  return launch_pdl(kPdlHook, balance_kernel<T, G, V, W, kDirect>, dim3(kDirect ? n_seg : p.units), dim3(32 * W), 0, s, static_cast<const T*>(logits),
                    ld, vec, idx, T_rows, E, k, act, seg, n_seg, p.unit_rows, part_p, part_c, part_n, out);
}
template <typename T>
cudaError_t balance_launch(const Plan& p, const void* logits, long long ld, const int* idx, int T_rows, int E, int k, int act, const int* seg,
                           int n_seg, float* part_p, int* part_c, int* part_n, const BalanceOut& out, cudaStream_t s) {
#define MIX_BALANCE_AS(G, V, W, D) \
  balance_launch_one<T, G, V, W, D>(p, logits, ld, idx, T_rows, E, k, act, seg, n_seg, part_p, part_c, part_n, out, s)
#define MIX_BALANCE(G, V)                                     \
  if (p.direct) return MIX_BALANCE_AS(G, V, kUnitWarps, true); \
  return p.warps == 1 ? MIX_BALANCE_AS(G, V, 1, false) : MIX_BALANCE_AS(G, V, kUnitWarps, false)
  MIX_ROW_LAYOUT(E, MIX_BALANCE);
#undef MIX_BALANCE
#undef MIX_BALANCE_AS
}
template <typename T>
cudaError_t grad_launch(const void* logits, long long ld, const int* idx, int T_rows, int E, int k, int act, const int* seg, int n_seg,
                        const int* counts, const int* rows, const float* d_loss, void* d_logits, long long ld_d, int n_sms, cudaStream_t s) {
  const int vec = (((uintptr_t)logits | (uintptr_t)(ld * (long long)sizeof(T))) & 15u) == 0;
  const int vec_d = (((uintptr_t)d_logits | (uintptr_t)(ld_d * (long long)sizeof(T))) & 15u) == 0;
  const int wave = 8 * kGradCtas * n_sms;                      // warps of one wave of CTAs
  int warp_rows = (int)(((long long)T_rows + wave - 1) / wave);
  if (warp_rows < 4) warp_rows = 4;
  const long long ctas = ((long long)T_rows + 8 * warp_rows - 1) / (8 * warp_rows);
#define MIX_BALANCE_GRAD(G, V)                                                                                                          \
  return launch_pdl(kPdlHook, balance_grad_kernel<T, G, V>, dim3((unsigned)ctas), dim3(256), 0, s, static_cast<const T*>(logits), ld, vec, \
                    idx, T_rows, E, k, act, seg, n_seg, counts, rows, d_loss, warp_rows, static_cast<T*>(d_logits), ld_d, vec_d)
  MIX_ROW_LAYOUT(E, MIX_BALANCE_GRAD);
#undef MIX_BALANCE_GRAD
}

int segment_args(const int* seg, int n_seg, char* errbuf, int errbuf_len) {
  if (n_seg < 1 || n_seg > MIX_BALANCE_MAX_SEGMENTS) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "n_seg %d outside [1, %d]", n_seg, MIX_BALANCE_MAX_SEGMENTS);
  if (!seg && n_seg != 1) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "without offsets there is one segment, not %d", n_seg);
  return MIX_OK;
}

}  // namespace

namespace mix {
int router_args(const void* logits, int dtype, long long ld, int T, int E, int k, int act, char* errbuf, int errbuf_len);
}

extern "C" long long mix_router_balance_workspace(int T, int n_experts, int n_seg) {
  if (T < 0 || T > kOpMaxRows || n_experts < 1 || n_experts > kOpMaxExperts || n_seg < 1 || n_seg > MIX_BALANCE_MAX_SEGMENTS) return MIX_ERR_OUT_OF_RANGE;
  int dev, n_sms;
  if (op_device(&dev, &n_sms) != cudaSuccess) {
    cudaGetLastError();
    return MIX_ERR_CUDA;
  }
  return workspace_bytes_of(plan(T, n_experts, n_seg, n_sms), n_experts);
}

extern "C" int mix_router_balance(const void* logits, int dtype, long long ld, const int* idx, int T, int n_experts, int k, int act,
                                  const int* seg, int n_seg, float* loss, int* counts, float* mean_p, int* rows, void* workspace,
                                  long long workspace_bytes, void* stream, char* errbuf, int errbuf_len) {
  int rc = router_args(logits, dtype, ld, T, n_experts, k, act, errbuf, errbuf_len);
  if (rc == MIX_OK) rc = segment_args(seg, n_seg, errbuf, errbuf_len);
  if (rc != MIX_OK) return rc;
  if ((T > 0 && !idx) || !loss || !counts || !mean_p || !rows) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "idx, loss, counts, mean_p and rows are required");
  if ((uintptr_t)workspace & 3u) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "the workspace is not on 4 bytes");
  int dev, n_sms;
  MIX_OP_CUDA(op_device(&dev, &n_sms));
  const Plan p = plan(T, n_experts, n_seg, n_sms);
  const long long need = workspace_bytes_of(p, n_experts);
  if (need > 0 && (!workspace || workspace_bytes < need)) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "the workspace has to hold %lld bytes", need);
  float* part_p = static_cast<float*>(workspace);
  int* part_c = reinterpret_cast<int*>(part_p + p.slots * n_experts);
  int* part_n = part_c + p.slots * n_experts;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const BalanceOut out = {loss, counts, mean_p, rows};
  if (T > 0 || p.direct) {
    cudaError_t e;
    if (dtype == MIX_DTYPE_F32) e = balance_launch<float>(p, logits, ld, idx, T, n_experts, k, act, seg, n_seg, part_p, part_c, part_n, out, s);
    else if (dtype == MIX_DTYPE_BF16) e = balance_launch<__nv_bfloat16>(p, logits, ld, idx, T, n_experts, k, act, seg, n_seg, part_p, part_c, part_n, out, s);
    else e = balance_launch<__half>(p, logits, ld, idx, T, n_experts, k, act, seg, n_seg, part_p, part_c, part_n, out, s);
    MIX_OP_CUDA(e);
  }
  if (p.direct) return MIX_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_seg * p.cluster));
  cfg.blockDim = dim3(p.warps == 1 && p.cluster == 1 ? ((n_experts + 31) & ~31) : kFinThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  int n_at = 0;
  if (p.cluster > 1) {
    at[n_at].id = cudaLaunchAttributeClusterDimension;
    at[n_at].val.clusterDim.x = p.cluster;
    at[n_at].val.clusterDim.y = 1;
    at[n_at++].val.clusterDim.z = 1;
  }
  if (pdl_mask() & kPdlHook) {
    at[n_at].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n_at++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = at;
  cfg.numAttrs = n_at;
  MIX_OP_CUDA(cudaLaunchKernelEx(&cfg, p.cluster > 1 ? balance_finish_kernel<kFinCluster, false> : (p.warps == 1 ? balance_finish_kernel<1, true> : balance_finish_kernel<1, false>), static_cast<const float*>(part_p),
                                 static_cast<const int*>(part_c), static_cast<const int*>(part_n), T, n_experts, seg, p.unit_rows, loss, counts,
                                 mean_p, rows));
  return MIX_OK;
}

extern "C" int mix_router_balance_grad(const void* logits, int dtype, long long ld, const int* idx, int T, int n_experts, int k, int act,
                                       const int* seg, int n_seg, const int* counts, const int* rows, const float* d_loss, void* d_logits,
                                       long long ld_d, void* stream, char* errbuf, int errbuf_len) {
  int rc = router_args(logits, dtype, ld, T, n_experts, k, act, errbuf, errbuf_len);
  if (rc == MIX_OK) rc = segment_args(seg, n_seg, errbuf, errbuf_len);
  if (rc != MIX_OK) return rc;
  if (ld_d < n_experts) MIX_OP_FAIL(MIX_ERR_OUT_OF_RANGE, "row stride %lld of d_logits is below n_experts %d", ld_d, n_experts);
  if (T == 0) return MIX_OK;
  if (!idx || !counts || !rows || !d_loss || !d_logits) MIX_OP_FAIL(MIX_ERR_INVALID_ARG, "idx, counts, rows, d_loss and d_logits are required");
  int dev, n_sms;
  MIX_OP_CUDA(op_device(&dev, &n_sms));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == MIX_DTYPE_F32) e = grad_launch<float>(logits, ld, idx, T, n_experts, k, act, seg, n_seg, counts, rows, d_loss, d_logits, ld_d, n_sms, s);
  else if (dtype == MIX_DTYPE_BF16) e = grad_launch<__nv_bfloat16>(logits, ld, idx, T, n_experts, k, act, seg, n_seg, counts, rows, d_loss, d_logits, ld_d, n_sms, s);
  else e = grad_launch<__half>(logits, ld, idx, T, n_experts, k, act, seg, n_seg, counts, rows, d_loss, d_logits, ld_d, n_sms, s);
  MIX_OP_CUDA(e);
  return MIX_OK;
}

// Tokens sorted by expert as rows of the caller's, and back (paper Sections 1 and 2.1: every token goes to its Top-K
// experts, whose outputs come back as a gate-weighted sum), with the gradients that training such a layer needs.  With
// p = t * top_k + j a pair and s(p) its place in the stable order by expert:
//   dispatch           rows[s(p)] = w[p] x[t]                    combine           y[t] = sum_j w[p] rows[s(p)]
//   dispatch_backward  dx[t] = sum_j w[p] drows[s(p)]            combine_backward  drows[s(p)] = w[p] dy[t]
//                      dw[p] = <x[t], drows[s(p)]>                                 dw[p] = <rows[s(p)], dy[t]>
// So there are two kernels: `spread` (a token's row to its pairs' rows) and `gather` (the pairs' rows to the token's), each with or
// without the k scalar products.  Both own whole tokens: a token's row is read or written once, however many picks it has,
// every sum has a fixed order, and the products need no atomics.
#include <cooperative_groups.h>

#include "rows.cuh"

namespace cg = cooperative_groups;

namespace emoe {
namespace {

constexpr int ROWS_THREADS = 256;
// CTAs per SM that the gather's registers are cut for: the rows in flight are what its speed goes by.  us without / with: 8192 tokens of 4096, two
// picks 37.3/35.2 (six; eight spill: 38.5), with products 61.7/48.0 (five; six 51.4); 16384 tokens of 2048, eight picks 113.9/99.2.
__host__ __device__ constexpr int gather_ctas(int picks, bool dots) { return picks >= 8 ? (dots ? 2 : 4) : picks == 2 && !dots ? 6 : 5; }
// ... and the spread's: 8192 tokens of 4096, two picks 40.2/38.3 (six / eight), with products 66.9/55.3; 16384 tokens of 2048, eight picks 122/116; with
// products, 8192 tokens, 117/98.
__host__ __device__ constexpr int spread_ctas(int picks, bool dots) { return dots ? (picks > 2 ? 3 : 5) : picks > 2 ? 5 : 8; }

struct RowsArgs {
  const void* in;    // spread: tokens; gather: rows
  const void* with;  // the other factor of the products: spread: rows, gather: tokens
  void* out;         // spread: rows; gather: tokens
  float* dots;       // [T][top_k]
  int32_t* perm;     // spread: written too (null: no)
  const int32_t* slots;
  const float* weights;  // null: 1
  int T, d, top_k, threads_per_token;
  int ahead, ahead_bytes;  // spread behind the sort: rounds of the first CTAs' tokens that are pulled to L2 meanwhile, bytes of a token
  size_t token_stride, row_stride;
};

// The pairs of one token: their rows and weights.  A dropped pair (slot outside [0, P)) has weight 0 and is neither read nor written.
template <int KM>
struct Pairs {
  int slot[KM];
  float w[KM];
  __device__ __forceinline__ void load(const RowsArgs& a, int t) {
#pragma unroll
    for (int j = 0; j < KM; ++j) {
      slot[j] = -1;
      w[j] = 0.f;
      if (j < a.top_k) {
        const size_t p = static_cast<size_t>(t) * a.top_k + j;
        const int s = a.slots[p];
        const float v = a.weights ? a.weights[p] : 1.f;
        if (s >= 0 && s < a.T * a.top_k) {
          slot[j] = s;
          w[j] = v;
        }
      }
    }
  }
};

// Adds a token's products over its threads (whole warps) and writes them.  Every thread of the CTA calls this.
template <int KM>
__device__ __forceinline__ void write_dots(const RowsArgs& a, float (&dot)[KM], int t, float (*s_dots)[KM]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int j = 0; j < KM; ++j)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
  if (lane == 0) {
#pragma unroll
    for (int j = 0; j < KM; ++j) s_dots[warp][j] = dot[j];
  }
  __syncthreads();
  const int in_token = threadIdx.x % a.threads_per_token;
  if (t < a.T && in_token < a.top_k) {
    const int warps = a.threads_per_token / 32;
    float sum = 0.f;
    for (int w = 0; w < warps; ++w) sum += s_dots[warp - in_token / 32 + w][in_token];
    a.dots[static_cast<size_t>(t) * a.top_k + in_token] = sum;
  }
}

// CTAs of the first round with one or two picks.  With more picks five of eight are resident while the sort runs, and the others pull their tokens just before
// they read them.
constexpr int SPREAD_FIRST = 8 * GPU_SMS;
__device__ __forceinline__ void prefetch_l2(const void* p, int bytes) {  // both multiples of 16
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

template <typename RowT, typename TokT, int VEC, int KM, bool DOTS>
__global__ void __launch_bounds__(ROWS_THREADS, spread_ctas(KM, DOTS)) spread_kernel(RowsArgs a) {
  __shared__ float s_dots[DOTS ? ROWS_THREADS / 32 : 1][KM];
  const int tpt = a.threads_per_token, in_token = threadIdx.x % tpt;
  const int t = blockIdx.x * (ROWS_THREADS / tpt) + threadIdx.x / tpt;
  if constexpr (!DOTS) {
    // While eight SMs sort, the others pull tokens to L2 (they are older than the sort, which waits before its trigger): of 200 MB read and
    // written the sort's 5 us hide some 30.
    if (blockIdx.x < SPREAD_FIRST && in_token == 0)
      for (int i = 0; i < a.ahead; ++i) {
        const int at = t + i * SPREAD_FIRST * (ROWS_THREADS / tpt);
        if (at < a.T) prefetch_l2(static_cast<const TokT*>(a.in) + static_cast<size_t>(at) * a.token_stride, a.ahead_bytes);
      }
  }
  pdl_wait();
  pdl_trigger();
  float dot[KM] = {};
  if (t < a.T) {
    Pairs<KM> pairs;
    pairs.load(a, t);
    if constexpr (!DOTS) {
      if (a.perm) {
#pragma unroll
        for (int j = 0; j < KM; ++j)
          if (in_token == j && pairs.slot[j] >= 0) a.perm[pairs.slot[j]] = t * a.top_k + j;
      }
    }
    const TokT* x = static_cast<const TokT*>(a.in) + static_cast<size_t>(t) * a.token_stride;
    constexpr int U = DOTS ? (KM > 2 ? 1 : 2) : VEC <= 2 ? 8 : 2;  // pieces asked for together
    for (int i0 = in_token * VEC; i0 < a.d; i0 += tpt * VEC * U) {
      Piece<TokT, VEC> px[U];
      Piece<RowT, VEC> pr[U][DOTS ? KM : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * tpt * VEC;
        if (i < a.d) px[u] = load_piece<TokT, VEC>(x + i);
        if constexpr (DOTS) {
#pragma unroll
          for (int j = 0; j < KM; ++j)
            if (i < a.d && pairs.slot[j] >= 0)
              pr[u][j] = load_piece<RowT, VEC>(static_cast<const RowT*>(a.with) + static_cast<size_t>(pairs.slot[j]) * a.row_stride + i);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * tpt * VEC;
        if (i >= a.d) break;
        float f[VEC];
        widen<TokT, VEC>(px[u], f);
#pragma unroll
        for (int j = 0; j < KM; ++j) {
          if (pairs.slot[j] < 0) continue;
          if constexpr (DOTS) {
            float r[VEC];
            widen<RowT, VEC>(pr[u][j], r);
#pragma unroll
            for (int v = 0; v < VEC; ++v) dot[j] = fmaf(r[v], f[v], dot[j]);
          }
          float o[VEC];
#pragma unroll
          for (int v = 0; v < VEC; ++v) o[v] = pairs.w[j] * f[v];
          store_piece<RowT, VEC>(static_cast<RowT*>(a.out) + static_cast<size_t>(pairs.slot[j]) * a.row_stride + i, narrow<RowT, VEC>(o));
        }
      }
    }
  }
  if constexpr (DOTS) write_dots<KM>(a, dot, t, s_dots);
}

template <typename RowT, typename TokT, int VEC, int KM, bool DOTS>
__global__ void __launch_bounds__(ROWS_THREADS, gather_ctas(KM, DOTS)) gather_kernel(RowsArgs a) {
  __shared__ float s_dots[DOTS ? ROWS_THREADS / 32 : 1][KM];
  pdl_wait();
  pdl_trigger();
  const int tpt = a.threads_per_token, in_token = threadIdx.x % tpt;
  const int t = blockIdx.x * (ROWS_THREADS / tpt) + threadIdx.x / tpt;
  float dot[KM] = {};
  if (t < a.T) {
    Pairs<KM> pairs;
    pairs.load(a, t);
    TokT* y = static_cast<TokT*>(a.out) + static_cast<size_t>(t) * a.token_stride;
    constexpr int U = KM == 1 ? 4 : KM == 2 && !(DOTS && VEC == 1) ? 2 : 1;  // pieces of every row asked for together
    for (int i0 = in_token * VEC; i0 < a.d; i0 += tpt * VEC * U) {
      Piece<RowT, VEC> pr[U][KM];
      Piece<TokT, VEC> px[DOTS ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * tpt * VEC;
#pragma unroll
        for (int j = 0; j < KM; ++j) {
          pr[u][j] = {};
          if (i < a.d && pairs.slot[j] >= 0)
            pr[u][j] = load_piece<RowT, VEC>(static_cast<const RowT*>(a.in) + static_cast<size_t>(pairs.slot[j]) * a.row_stride + i);
        }
        if constexpr (DOTS)
          if (i < a.d) px[u] = load_piece<TokT, VEC>(static_cast<const TokT*>(a.with) + static_cast<size_t>(t) * a.token_stride + i);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * tpt * VEC;
        if (i >= a.d) break;
        float sum[VEC] = {}, x[DOTS ? VEC : 1];
        if constexpr (DOTS) widen<TokT, VEC>(px[u], x);
#pragma unroll
        for (int j = 0; j < KM; ++j) {
          if (pairs.slot[j] < 0) continue;
          float r[VEC];
          widen<RowT, VEC>(pr[u][j], r);
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            sum[v] = fmaf(pairs.w[j], r[v], sum[v]);
            if constexpr (DOTS) dot[j] = fmaf(r[v], x[v], dot[j]);
          }
        }
        store_piece<TokT, VEC>(y + i, narrow<TokT, VEC>(sum));
      }
    }
  }
  if constexpr (DOTS) write_dots<KM>(a, dot, t, s_dots);
}

// ---- the order --------------------------------------------------------------------------------

// Stable counting sort by one cluster of up to eight CTAs.  A warp owns a run of consecutive pairs: it counts them by expert, the counts of all warps in front of it, of its CTA and of the CTAs before (read
// over distributed shared memory), are its first places, and a second walk hands them out.  Two cluster-wide waits,
// no order-dependent atomics.  keep_rest: ids outside [0, E - 1) count as E - 1.
constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32, SORT_CLUSTER = 8, SORT_STEPS = 16;

__global__ void __launch_bounds__(SORT_THREADS)
    sort_pairs_kernel(const int32_t* __restrict__ ids, int n, int E, bool keep_rest, int32_t* __restrict__ counts, int32_t* __restrict__ off,
                      int32_t* __restrict__ perm, bool write_perm, int32_t* __restrict__ slot_of_pair, int* __restrict__ check_word) {
  extern __shared__ int first[];  // [SORT_WARPS][E]: pairs of a warp by expert, then the next place of each
  __shared__ int hist[EMOE_MAX_EXPERTS + 1], s_off[EMOE_MAX_EXPERTS + 2];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster.block_rank()), ctas = static_cast<int>(cluster.num_blocks());
  const int run = (n + ctas * SORT_THREADS - 1) / (ctas * SORT_THREADS) * 32;
  const int begin = (rank * SORT_WARPS + warp) * run;
  int* mine = first + warp * E;
  const int bits = 32 - __clz(E - 1 > 0 ? E - 1 : 1);
  const int named = keep_rest ? E - 1 : E, rest = keep_rest ? E - 1 : -1;
  for (int i = tid; i < SORT_WARPS * E; i += SORT_THREADS) first[i] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  bool bad = false;
  // Ids of sixteen steps are asked for together.  A step's lanes of one expert come from one ballot per bit of the id (match.any takes a
  // round per different value: 43 us instead of 9 for 131072 pairs of 128 experts).  place: rank among them and, in the first of them, how many.
  int id[SORT_STEPS], place[SORT_STEPS];
  const auto load = [&](int p0) {
#pragma unroll
    for (int i = 0; i < SORT_STEPS; ++i) {
      const int p = p0 + 32 * i + lane;
      const bool live = 32 * i < run - (p0 - begin) && p < n;
      id[i] = live ? ids[p] : -1;
      if (live && (id[i] < 0 || id[i] >= named)) {
        bad |= !keep_rest || id[i] != -1;
        id[i] = rest;
      }
    }
#pragma unroll
    for (int i = 0; i < SORT_STEPS; ++i) {
      if (p0 + 32 * i >= begin + run || p0 + 32 * i >= n) break;
      unsigned same = __ballot_sync(0xffffffffu, id[i] >= 0);
      for (int b = 0; b < bits; ++b) {
        const unsigned set = __ballot_sync(0xffffffffu, id[i] >> b & 1);
        same &= (id[i] >> b & 1) ? set : ~set;
      }
      const int rank_in = __popc(same & ((1u << lane) - 1u));
      place[i] = rank_in == 0 ? __popc(same) << 8 : rank_in;
    }
  };
  for (int p0 = begin; p0 < begin + run && p0 < n; p0 += 32 * SORT_STEPS) {
    load(p0);
#pragma unroll
    for (int i = 0; i < SORT_STEPS; ++i) {
      if (p0 + 32 * i >= begin + run || p0 + 32 * i >= n) break;
      if (id[i] >= 0 && place[i] >= 256) mine[id[i]] += place[i] >> 8;
      __syncwarp();
    }
  }
  if (bad) atomicOr(check_word, CHECK_BAD_EXPERT_ID);
  __syncthreads();
  if (tid < E) {
    int sum = 0;
#pragma unroll 8
    for (int w = 0; w < SORT_WARPS; ++w) sum += first[w * E + tid];
    hist[tid] = sum;
  }
  cluster.sync();
  int before = 0, total = 0;
  if (tid < E) {
    int of_cta[SORT_CLUSTER];
#pragma unroll
    for (int r = 0; r < SORT_CLUSTER; ++r) of_cta[r] = r < ctas ? cluster.map_shared_rank(hist, r)[tid] : 0;
#pragma unroll
    for (int r = 0; r < SORT_CLUSTER; ++r) {
      if (r < rank) before += of_cta[r];
      total += of_cta[r];
    }
    s_off[tid + 1] = total;
    if (rank == 0 && counts) counts[tid] = total;
  }
  __syncthreads();
  if (warp == 0) {
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + lane;
      int incl = e < E ? s_off[e + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (e < E) s_off[e + 1] = carry + incl;
      carry += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) s_off[0] = 0;
  }
  __syncthreads();
  if (tid < E) {
    int next = s_off[tid] + before;
    for (int w0 = 0; w0 < SORT_WARPS; w0 += 8) {
      int c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = first[(w0 + w) * E + tid];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        first[(w0 + w) * E + tid] = next;
        next += c[w];
      }
    }
  }
  if (rank == 0)
    for (int e = tid; e <= E; e += SORT_THREADS) off[e] = s_off[e];
  // pairs without an expert own no place: what lies behind the last one reads as "no pair"
  for (int p = s_off[E] + rank * SORT_THREADS + tid; p < n; p += ctas * SORT_THREADS) perm[p] = -1;
  __syncthreads();
  for (int p0 = begin; p0 < begin + run && p0 < n; p0 += 32 * SORT_STEPS) {
    if (run > 32 * SORT_STEPS) load(p0);
#pragma unroll
    for (int i = 0; i < SORT_STEPS; ++i) {
      if (p0 + 32 * i >= begin + run || p0 + 32 * i >= n) break;
      const int p = p0 + 32 * i + lane, e = id[i];
      int pos = -1;
      if (e >= 0) {
        pos = mine[e] + (place[i] & 255);
        if (write_perm) perm[pos] = p;
      }
      if (p < n && slot_of_pair) slot_of_pair[p] = pos;
      __syncwarp();
      if (e >= 0 && place[i] >= 256) mine[e] += place[i] >> 8;
      __syncwarp();
    }
  }
  cluster.sync();  // nobody leaves while another CTA reads its counts
}

// Few pairs: order and rows in one launch.  A CTA per token counts, for each of its pairs, the pairs in front of it in the order (all ids,
// from L2) while its row is on the way; one CTA more writes counts, offsets and the places of no pair.  us, order by the cluster and rows behind
// it / this, tokens of 4096, two picks: 64 tokens 5.3/2.0, 512 tokens 7.6/3.8, 1024 tokens 9.4/6.1, 2048 tokens 14.6/15.0.
constexpr int DISPATCH_ONE_PAIRS = 2048;
template <typename RowT, typename TokT, int VEC, int KM>
__global__ void __launch_bounds__(ROWS_THREADS)
    dispatch_one_kernel(RowsArgs a, const int32_t* __restrict__ ids, int E, int32_t* __restrict__ counts, int32_t* __restrict__ off,
                        int32_t* __restrict__ perm, int32_t* __restrict__ slot_of_pair, int* __restrict__ check_word) {
  __shared__ int s_cnt[EMOE_MAX_EXPERTS + 1];
  __shared__ int s_part[ROWS_THREADS / 32][KM];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, P = a.T * a.top_k;
  pdl_wait();
  pdl_trigger();
  if (static_cast<int>(blockIdx.x) == a.T) {
    for (int e = tid; e <= E; e += ROWS_THREADS) s_cnt[e] = 0;
    __syncthreads();
    bool bad = false;
    for (int p = tid; p < P; p += ROWS_THREADS) {
      const int e = ids[p];
      if (e >= 0 && e < E) atomicAdd(&s_cnt[e + 1], 1);
      else {
        bad = true;
        slot_of_pair[p] = -1;
      }
    }
    if (bad) atomicOr(check_word, CHECK_BAD_EXPERT_ID);
    __syncthreads();
    if (warp == 0) {
      int carry = 0;
      for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane, c = e < E ? s_cnt[e + 1] : 0;
        int incl = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += v;
        }
        if (e < E) {
          counts[e] = c;
          off[e] = carry + incl - c;
        }
        carry += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (lane == 0) {
        off[E] = carry;
        s_cnt[0] = carry;
      }
    }
    __syncthreads();
    for (int p = s_cnt[0] + tid; p < P; p += ROWS_THREADS) perm[p] = -1;
    return;
  }
  const int t = blockIdx.x;
  const TokT* x = static_cast<const TokT*>(a.in) + static_cast<size_t>(t) * a.token_stride;
  constexpr int U = VEC <= 2 ? 8 : 2;  // pieces asked for together (narrow ones, two / eight: 2000 x 5001, one pick 27/22, 60 x 1101, two picks 2.4/1.9)
  Piece<TokT, VEC> px[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if ((tid + u * ROWS_THREADS) * VEC < a.d) px[u] = load_piece<TokT, VEC>(x + (tid + u * ROWS_THREADS) * VEC);
  int e[KM], in_front[KM];
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    in_front[j] = 0;
    e[j] = j < a.top_k ? ids[t * a.top_k + j] : -1;
    if (e[j] >= E) e[j] = -1;
  }
  for (int q = tid; q < P; q += ROWS_THREADS) {
    const int eq = ids[q];
    if (eq < 0 || eq >= E) continue;
#pragma unroll
    for (int j = 0; j < KM; ++j)
      if (j < a.top_k) in_front[j] += eq < e[j] || (eq == e[j] && q < t * a.top_k + j);
  }
#pragma unroll
  for (int j = 0; j < KM; ++j)
    if (j < a.top_k) {
      const int sum = __reduce_add_sync(0xffffffffu, in_front[j]);
      if (lane == 0) s_part[warp][j] = sum;
    }
  __syncthreads();
  int slot[KM];
  float w[KM];
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    slot[j] = -1;
    w[j] = 1.f;
    if (j < a.top_k && e[j] >= 0) {
      int s = 0;
#pragma unroll
      for (int i = 0; i < ROWS_THREADS / 32; ++i) s += s_part[i][j];
      slot[j] = s;
      const int p = t * a.top_k + j;
      if (a.weights) w[j] = a.weights[p];
      if (tid == j) {
        perm[s] = p;
        slot_of_pair[p] = s;
      }
    }
  }
  for (int i0 = tid * VEC, first = 1; i0 < a.d; i0 += ROWS_THREADS * VEC * U, first = 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * ROWS_THREADS * VEC;
      if (i >= a.d) break;
      if (!first) px[u] = load_piece<TokT, VEC>(x + i);
      float f[VEC];
      widen<TokT, VEC>(px[u], f);
#pragma unroll
      for (int j = 0; j < KM; ++j) {
        if (slot[j] < 0) continue;
        float o[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) o[v] = w[j] * f[v];
        store_piece<RowT, VEC>(static_cast<RowT*>(a.out) + static_cast<size_t>(slot[j]) * a.row_stride + i, narrow<RowT, VEC>(o));
      }
    }
  }
}

// ---- gradient of the gates ----------------------------------------------------------------------

// dz from the gradient of the Top-K gates.  LANES neighbouring lanes own a token, each V of its logits: V runs of LANES
// neighbours, or (VEC4) runs of four.  Softmax over all experts: g_j = p_{i_j}, so
//   dz_e = p_e (D_e - sum_e' D_e' p_e'),  D_e = sum of the dg_j whose pick is e.
// Renormalised over the picks: g is a softmax over the picked logits alone (the other experts cancel), dz is zero elsewhere and
// only the picks' logits are read.
template <int LANES, int V, bool VEC4, bool RENORM>
__global__ void __launch_bounds__(256)
    gate_backward_kernel(const float* __restrict__ logits, int T, int E, const int32_t* __restrict__ ids, const float* __restrict__ dgates,
                         int top_k, float* __restrict__ dlogits, int* __restrict__ check_word) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % LANES;
  const int t = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (__all_sync(0xffffffffu, t >= T)) return;
  const bool live = t < T;
  const float* z = logits + static_cast<size_t>(live ? t : 0) * E;
  const auto at = [&](int i) { return VEC4 ? (i / 4) * LANES * 4 + lane * 4 + i % 4 : i * LANES + lane; };
  const auto group_max = [](float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  };
  const auto group_sum = [](float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  // lane j holds pick j
  int pick = -1;
  float dg = 0.f;
  if (live && lane < top_k) {
    pick = ids[static_cast<size_t>(t) * top_k + lane];
    dg = dgates[static_cast<size_t>(t) * top_k + lane];
    if (pick < 0 || pick >= E) {
      atomicOr(check_word, CHECK_BAD_EXPERT_ID);
      pick = -1;
      dg = 0.f;
    }
  }
  float out[V];
  if constexpr (RENORM) {
    const float zj = pick >= 0 ? z[pick] : -INFINITY;
    const float top = group_max(zj);
    float g = pick >= 0 && top > -INFINITY ? expf(zj - top) : 0.f;
    if (pick >= 0 && isnan(zj)) g = zj;
    const float sum = group_sum(g);
    g = sum != 0.f ? g / sum : 0.f;
    const float c = group_sum(pick >= 0 ? g * dg : 0.f);
    const float dz = sum != 0.f ? g * (dg - c) : 0.f;  // (no logit left: zero, whatever dg is)
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = 0.f;
    for (int j = 0; j < top_k; ++j) {
      const int e = __shfl_sync(0xffffffffu, pick, j, LANES);
      const float v = __shfl_sync(0xffffffffu, dz, j, LANES);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (at(i) == e) out[i] += v;
    }
  } else {
    float p[V];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = -INFINITY;
    if (live) {
      if constexpr (VEC4) {
#pragma unroll
        for (int i = 0; i < V; i += 4)
          if (at(i) < E) {
            const float4 q = *reinterpret_cast<const float4*>(z + at(i));
            p[i] = q.x; p[i + 1] = q.y; p[i + 2] = q.z; p[i + 3] = q.w;
          }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (at(i) < E) p[i] = z[at(i)];
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) top = fmaxf(top, p[i]);
    top = group_max(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // a row of nothing but -inf has no softmax: its gradient is zero
      if (!isnan(p[i])) p[i] = top > -INFINITY ? expf(p[i] - top) : 0.f;
      sum += p[i];
      out[i] = 0.f;
    }
    sum = group_sum(sum);
    for (int j = 0; j < top_k; ++j) {
      const int e = __shfl_sync(0xffffffffu, pick, j, LANES);
      const float v = __shfl_sync(0xffffffffu, dg, j, LANES);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (at(i) == e) out[i] += v;
    }
    float c = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      p[i] = sum != 0.f ? p[i] / sum : 0.f;
      c = fmaf(p[i], out[i], c);
    }
    c = group_sum(c);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = sum != 0.f ? p[i] * (out[i] - c) : 0.f;
  }
  if (!live) return;
  float* dz = dlogits + static_cast<size_t>(t) * E;
  if constexpr (VEC4) {
#pragma unroll
    for (int i = 0; i < V; i += 4)
      if (at(i) < E) *reinterpret_cast<float4*>(dz + at(i)) = make_float4(out[i], out[i + 1], out[i + 2], out[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at(i) < E) dz[at(i)] = out[i];
  }
}

// ---- launches -----------------------------------------------------------------------------------

template <typename T>
struct Tag {
  using type = T;
};

// f(rows' type, tokens' type, values per piece): 16 bytes of a row where every address and the row length allow them, else two values, else one
enum Width { ONE, TWO, WIDE };
template <typename F>
cudaError_t by_types(int row_dtype, int token_dtype, Width width, F&& f) {
  const auto by_width = [&](auto row, auto tok) -> cudaError_t {
    constexpr int MOST = sizeof(typename decltype(row)::type) == 2 ? 8 : 4;
    if (width == WIDE) return f(row, tok, std::integral_constant<int, MOST>());
    return width == TWO ? f(row, tok, std::integral_constant<int, 2>()) : f(row, tok, std::integral_constant<int, 1>());
  };
  const bool tb = token_dtype == EMOE_DTYPE_BF16;
  if (row_dtype == EMOE_DTYPE_BF16) return tb ? by_width(Tag<__nv_bfloat16>(), Tag<__nv_bfloat16>()) : by_width(Tag<__nv_bfloat16>(), Tag<float>());
  return tb ? by_width(Tag<float>(), Tag<__nv_bfloat16>()) : by_width(Tag<float>(), Tag<float>());
}

// Threads of a token, by the pieces of its row.  Wide pieces: as few as take the row in one `round` of pieces asked for together, while that
// leaves work for 64 K threads, and as leave each `most` times 16 bytes (of the wider type), while that fills the SMs (`ctas` each): rows in flight hide more
// than threads on one row.  us, a thread per piece / as ruled: combine 8192 x 1024, one pick 9.7/5.8, 8192 x 2048, two picks 24.5/18.1; its gradient,
// 30000 x 512, one pick 28.4/19.4; 1100 x 1024, two picks 2.9/2.2 (32 threads 2.8); 300 x 1024, eight picks 2.8 with 128 threads, 5.0 with
// 32.  Narrower pieces: about a thread per 16 bytes (combine 8192 x 1101, two picks, 32 / 64 / 128 / 256 threads 30.7/25.5/26.4/31.3; 4000 x 777,
// eight picks 34.5/37.0/31.5/35.1).  Over 92 calls 12 % less than a thread per piece, 2 % more than the best.
int threads_per_token(const emoe_dispatch_desc& D, int T, Width width, int round, int most, int ctas) {
  const size_t size = D.row_dtype == EMOE_DTYPE_BF16 && D.token_dtype == EMOE_DTYPE_BF16 ? 2 : 4;
  const long long words = static_cast<long long>((D.d * size + 15) / 16), pieces = D.row_dtype == EMOE_DTYPE_BF16 ? (D.d + 7) / 8 : (D.d + 3) / 4;
  int t = 32;
  if (width != WIDE) {
    while (t < ROWS_THREADS && 2LL * t * t < words * words) t *= 2;
    return t;
  }
  while (t < ROWS_THREADS && t < pieces) t *= 2;
  const auto halves = [&](int each, long long of, long long threads) {
    return t > 32 && static_cast<long long>(t / 2) * each >= of && static_cast<long long>(T) * (t / 2) >= threads;
  };
  while (halves(round, pieces, 1 << 16) || halves(most, words, static_cast<long long>(ctas) * ROWS_THREADS * GPU_SMS)) t /= 2;
  return t;
}
int gather_threads(const emoe_dispatch_desc& D, const RowsArgs& a, Width width) {
  const int picks = a.top_k <= 2 ? (a.dots ? 2 : a.top_k) : a.top_k <= 4 && !a.dots ? 4 : 8;
  const bool widens = D.row_dtype == EMOE_DTYPE_BF16 && D.token_dtype == EMOE_DTYPE_F32;  // (2048 x 1024, one pick, 32 / 64 / 128 threads 4.3/4.8/3.6 us)
  return threads_per_token(D, a.T, width, picks > 2 || (picks == 1 && widens) ? 1 : picks == 1 ? 4 : 2, 4, gather_ctas(picks, a.dots));
}
// (a spread writes top_k rows per piece: 4000 x 2048, eight picks, two / four pieces 30.8/35.0, with products 47.1/49.7)
int spread_threads(const emoe_dispatch_desc& D, const RowsArgs& a, Width width) {
  return threads_per_token(D, a.T, width, a.dots && a.top_k > 2 ? 1 : 2, a.dots && a.top_k <= 2 ? 4 : 2, spread_ctas(a.top_k <= 2 ? 2 : 8, a.dots));
}

Width width_of(const emoe_dispatch_desc& D, const RowsArgs& a, const void* rows, const void* rows_too, const void* tokens, const void* tokens_too) {
  const size_t rz = dtype_size(D.row_dtype), tz = dtype_size(D.token_dtype);
  const auto fits = [&](int vec) {
    const size_t ra = vec * rz < 16 ? vec * rz : 16, ta = vec * tz < 16 ? vec * tz : 16;
    return a.d % vec == 0 && a.row_stride * rz % ra == 0 && a.token_stride * tz % ta == 0 && ptr_aligned(rows, ra) && ptr_aligned(rows_too, ra) &&
           ptr_aligned(tokens, ta) && ptr_aligned(tokens_too, ta);
  };
  return fits(rz == 2 ? 8 : 4) ? WIDE : fits(2) ? TWO : ONE;
}

cudaError_t launch_gather(const emoe_dispatch_desc& D, RowsArgs a, cudaStream_t st) {
  const Width wide = width_of(D, a, a.in, nullptr, a.out, a.with);
  return by_types(D.row_dtype, D.token_dtype, wide, [&](auto row, auto tok, auto vec) {
    using RowT = typename decltype(row)::type;
    using TokT = typename decltype(tok)::type;
    constexpr int VEC = decltype(vec)::value;
    a.threads_per_token = gather_threads(D, a, wide);
    const int per_cta = ROWS_THREADS / a.threads_per_token;
    const auto go = [&](auto kernel) { return launch_chain(kernel, dim3((a.T + per_cta - 1) / per_cta), dim3(ROWS_THREADS), 0, st, a); };
    if (a.dots) return a.top_k <= 2 ? go(gather_kernel<RowT, TokT, VEC, 2, true>) : go(gather_kernel<RowT, TokT, VEC, 8, true>);
    if (a.top_k == 1) return go(gather_kernel<RowT, TokT, VEC, 1, false>);
    if (a.top_k == 2) return go(gather_kernel<RowT, TokT, VEC, 2, false>);
    return a.top_k <= 4 ? go(gather_kernel<RowT, TokT, VEC, 4, false>) : go(gather_kernel<RowT, TokT, VEC, 8, false>);
  });
}

// the picks known: slots given
cudaError_t launch_spread(const emoe_dispatch_desc& D, RowsArgs a, cudaStream_t st) {
  const Width wide = width_of(D, a, a.out, a.with, a.in, nullptr);
  return by_types(D.row_dtype, D.token_dtype, wide, [&](auto row, auto tok, auto vec) {
    using RowT = typename decltype(row)::type;
    using TokT = typename decltype(tok)::type;
    constexpr int VEC = decltype(vec)::value;
    a.threads_per_token = spread_threads(D, a, wide);
    const int per_cta = ROWS_THREADS / a.threads_per_token;
    const auto go = [&](auto kernel) { return launch_chain(kernel, dim3((a.T + per_cta - 1) / per_cta), dim3(ROWS_THREADS), 0, st, a); };
    if (a.dots) return a.top_k <= 2 ? go(spread_kernel<RowT, TokT, VEC, 2, true>) : go(spread_kernel<RowT, TokT, VEC, 8, true>);
    return a.top_k <= 2 ? go(spread_kernel<RowT, TokT, VEC, 2, false>) : go(spread_kernel<RowT, TokT, VEC, 8, false>);
  });
}

cudaError_t launch_dispatch_one(const emoe_dispatch_desc& D, RowsArgs a, const int32_t* ids, int32_t* counts, int32_t* off, int32_t* perm,
                                int32_t* slots, int* check_word, cudaStream_t st) {
  const Width wide = width_of(D, a, a.out, nullptr, a.in, nullptr);
  return by_types(D.row_dtype, D.token_dtype, wide, [&](auto row, auto tok, auto vec) {
    using RowT = typename decltype(row)::type;
    using TokT = typename decltype(tok)::type;
    const auto go = [&](auto kernel) {
      return launch_chain(kernel, dim3(a.T + 1), dim3(ROWS_THREADS), 0, st, a, ids, D.n_experts, counts, off, perm, slots, check_word);
    };
    return a.top_k <= 2 ? go(dispatch_one_kernel<RowT, TokT, decltype(vec)::value, 2>) : go(dispatch_one_kernel<RowT, TokT, decltype(vec)::value, 8>);
  });
}

template <int LANES, int V>
cudaError_t launch_gate(bool vec4, bool renorm, const float* z, int T, int E, const int32_t* ids, const float* dg, int top_k, float* dz, int* check,
                        cudaStream_t st) {
  const auto go = [&](auto kernel) {
    return launch_chain(kernel, dim3((T + 256 / LANES - 1) / (256 / LANES)), dim3(256), 0, st, z, T, E, ids, dg, top_k, dz, check);
  };
  if (vec4) return renorm ? go(gate_backward_kernel<LANES, V, true, true>) : go(gate_backward_kernel<LANES, V, true, false>);
  return renorm ? go(gate_backward_kernel<LANES, V, false, true>) : go(gate_backward_kernel<LANES, V, false, false>);
}

int check_dispatch(const emoe_dispatch_desc* D, int T, RowsArgs* a) {
  if (!D || T <= 0 || D->d <= 0) return EMOE_ERR_INVALID_ARG;
  if (D->n_experts < 1 || D->n_experts > EMOE_MAX_EXPERTS || D->top_k < 1 || D->top_k > EMOE_MAX_TOP_K) return EMOE_ERR_INVALID_ARG;
  if (D->token_stride < 0 || D->row_stride < 0) return EMOE_ERR_INVALID_ARG;
  if ((D->token_stride && D->token_stride < D->d) || (D->row_stride && D->row_stride < D->d)) return EMOE_ERR_INVALID_ARG;
  if (!dtype_ok(D->token_dtype) || !dtype_ok(D->row_dtype)) return EMOE_ERR_UNSUPPORTED;
  if (static_cast<long long>(T) * D->top_k > 0x7fffffffLL / 4 || D->d > 0x7fffffff / 64) return EMOE_ERR_UNSUPPORTED;
  *a = {};
  a->T = T;
  a->d = D->d;
  a->top_k = D->top_k;
  a->token_stride = static_cast<size_t>(D->token_stride ? D->token_stride : D->d);
  a->row_stride = static_cast<size_t>(D->row_stride ? D->row_stride : D->d);
  return EMOE_OK;
}

bool elements_aligned(const emoe_dispatch_desc* D, const void* tokens, const void* rows) {
  return ptr_aligned(tokens, dtype_size(D->token_dtype)) && ptr_aligned(rows, dtype_size(D->row_dtype));
}

// indices and fp32 vectors (null: not given)
template <typename... P>
bool words_aligned(const P*... p) {
  return (ptr_aligned(p, 4) && ...);
}

}  // namespace

cudaError_t launch_sort_pairs(const int32_t* ids, int n, int E, bool rest, int32_t* counts, int32_t* off, int32_t* perm, bool write_perm, int32_t* slot_of_pair,
                              int* check_word, cudaStream_t st) {
  const int ctas = n <= 2 * SORT_THREADS ? 1 : SORT_CLUSTER;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(SORT_THREADS);
  cfg.dynamicSmemBytes = sizeof(int) * SORT_WARPS * E;
  cfg.stream = st;
  static_assert(sizeof(int) * (SORT_WARPS + 2) * (EMOE_MAX_EXPERTS + 1) + 64 <= 48 * 1024, "no larger limit is asked for");
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {static_cast<unsigned>(ctas), 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl_enabled ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, sort_pairs_kernel, ids, n, E, rest, counts, off, perm, write_perm, slot_of_pair, check_word);
}

}  // namespace emoe

using namespace emoe;

#define EMOE_CALL(ctx, call)                                    \
  do {                                                          \
    const cudaError_t e__ = (call);                             \
    if (e__ != cudaSuccess) return ctx_cuda_fail(ctx, e__);     \
  } while (0)

extern "C" {

int emoe_dispatch(emoe_ctx* ctx, const emoe_dispatch_desc* desc, const void* x, int T, const int32_t* ids, const float* weights,
                  int32_t* out_counts, int32_t* out_off, int32_t* out_perm, int32_t* out_slot_of_pair, void* out_rows, void* stream) {
  RowsArgs a;
  const int rc = check_dispatch(desc, T, &a);
  if (rc != EMOE_OK) return rc;
  if (!x || !ids || !out_counts || !out_off || !out_perm || !out_slot_of_pair || !out_rows) return EMOE_ERR_INVALID_ARG;
  if (!elements_aligned(desc, x, out_rows) || !words_aligned(ids, weights, out_counts, out_off, out_perm, out_slot_of_pair)) return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.in = x;
  a.out = out_rows;
  a.weights = weights;
  a.slots = out_slot_of_pair;
  if (T * desc->top_k <= DISPATCH_ONE_PAIRS) {
    EMOE_CALL(ctx, launch_dispatch_one(*desc, a, ids, out_counts, out_off, out_perm, out_slot_of_pair, ctx_check_word(ctx), st));
    return EMOE_OK;
  }
  EMOE_CALL(ctx, launch_sort_pairs(ids, T * desc->top_k, desc->n_experts, false, out_counts, out_off, out_perm, false,
                                   out_slot_of_pair, ctx_check_word(ctx), st));
  a.perm = out_perm;  // scattered words: from all SMs, not from the eight of the sort
  const size_t z = dtype_size(desc->token_dtype), bytes = desc->d * z;
  if (bytes % 16 == 0 && a.token_stride * z % 16 == 0 && ptr_aligned(x, 16) && bytes <= (1 << 20)) {
    // some 32 MB, a quarter of L2
    const int threads = spread_threads(*desc, a, width_of(*desc, a, a.out, nullptr, a.in, nullptr));
    const size_t round = bytes * SPREAD_FIRST * (ROWS_THREADS / threads), rounds = (32u << 20) / round;
    a.ahead = rounds < 1 ? 1 : rounds < 16 ? static_cast<int>(rounds) : 16;
    a.ahead_bytes = static_cast<int>(bytes);
  }
  EMOE_CALL(ctx, launch_spread(*desc, a, st));
  return EMOE_OK;
}

int emoe_dispatch_backward(emoe_ctx* ctx, const emoe_dispatch_desc* desc, const void* drows, int T, const int32_t* slot_of_pair,
                           const float* weights, const void* x, void* dx, float* dweights, void* stream) {
  RowsArgs a;
  const int rc = check_dispatch(desc, T, &a);
  if (rc != EMOE_OK) return rc;
  if (!drows || !slot_of_pair || !dx) return EMOE_ERR_INVALID_ARG;
  if (dweights && !x) return EMOE_ERR_INVALID_ARG;
  if (!elements_aligned(desc, dx, drows) || (dweights && !elements_aligned(desc, x, drows)) || !words_aligned(slot_of_pair, weights, dweights)) return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  a.in = drows;
  a.with = dweights ? x : nullptr;
  a.out = dx;
  a.dots = dweights;
  a.slots = slot_of_pair;
  a.weights = weights;
  EMOE_CALL(ctx, launch_gather(*desc, a, static_cast<cudaStream_t>(stream)));
  return EMOE_OK;
}

int emoe_combine(emoe_ctx* ctx, const emoe_dispatch_desc* desc, const void* rows, int T, const int32_t* slot_of_pair, const float* gates, void* y,
                 void* stream) {
  RowsArgs a;
  const int rc = check_dispatch(desc, T, &a);
  if (rc != EMOE_OK) return rc;
  if (!rows || !slot_of_pair || !y) return EMOE_ERR_INVALID_ARG;
  if (!elements_aligned(desc, y, rows) || !words_aligned(slot_of_pair, gates)) return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  a.in = rows;
  a.out = y;
  a.slots = slot_of_pair;
  a.weights = gates;
  EMOE_CALL(ctx, launch_gather(*desc, a, static_cast<cudaStream_t>(stream)));
  return EMOE_OK;
}

int emoe_combine_backward(emoe_ctx* ctx, const emoe_dispatch_desc* desc, const void* dy, int T, const int32_t* slot_of_pair, const float* gates,
                          const void* rows, void* drows, float* dgates, void* stream) {
  RowsArgs a;
  const int rc = check_dispatch(desc, T, &a);
  if (rc != EMOE_OK) return rc;
  if (!dy || !slot_of_pair || !drows || (dgates && !rows)) return EMOE_ERR_INVALID_ARG;
  if (!elements_aligned(desc, dy, drows) || (dgates && !elements_aligned(desc, dy, rows)) || !words_aligned(slot_of_pair, gates, dgates)) return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  a.in = dy;
  a.with = dgates ? rows : nullptr;
  a.out = drows;
  a.dots = dgates;
  a.slots = slot_of_pair;
  a.weights = gates;
  EMOE_CALL(ctx, launch_spread(*desc, a, static_cast<cudaStream_t>(stream)));
  return EMOE_OK;
}

int emoe_gate_backward(emoe_ctx* ctx, const float* logits, int T, int E, const int32_t* ids, const float* dgates, int top_k, int gate_mode,
                       float* dlogits, void* stream) {
  if (!logits || !ids || !dgates || !dlogits || T <= 0) return EMOE_ERR_INVALID_ARG;
  if (E < 1 || E > EMOE_MAX_EXPERTS || top_k < 1 || top_k > E || top_k > EMOE_MAX_TOP_K) return EMOE_ERR_INVALID_ARG;
  if (gate_mode != EMOE_GATE_SOFTMAX && gate_mode != EMOE_GATE_SOFTMAX_RENORM) return EMOE_ERR_UNSUPPORTED;
  if (T > 0x7fffffff / 4) return EMOE_ERR_UNSUPPORTED;
  if (!words_aligned(logits, ids, dgates, dlogits)) return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool renorm = gate_mode == EMOE_GATE_SOFTMAX_RENORM, vec4 = E % 4 == 0 && ptr_aligned(logits, 16) && ptr_aligned(dlogits, 16);
  int* check = ctx_check_word(ctx);
  // eight lanes hold the picks of the widest gate; four logits per lane, eight beyond 128 experts
  if (E <= 32) EMOE_CALL(ctx, (launch_gate<8, 4>(vec4, renorm, logits, T, E, ids, dgates, top_k, dlogits, check, st)));
  else if (E <= 64) EMOE_CALL(ctx, (launch_gate<16, 4>(vec4, renorm, logits, T, E, ids, dgates, top_k, dlogits, check, st)));
  else if (E <= 128) EMOE_CALL(ctx, (launch_gate<32, 4>(vec4, renorm, logits, T, E, ids, dgates, top_k, dlogits, check, st)));
  else EMOE_CALL(ctx, (launch_gate<32, 8>(vec4, renorm, logits, T, E, ids, dgates, top_k, dlogits, check, st)));
  return EMOE_OK;
}

}  // extern "C"

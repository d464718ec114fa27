// Low-rank adapters of many requests (or experts) beside a shared projection, and their gradient.  Row i of a call belongs to
// adapter a(i) with factors A_a [rank][in], B_a [out][rank] and scale s_a:
//   forward   v_i = A_a x_i,                       y_i  = base_i + s_a B_a v_i
//   backward  dv_i = s_a B_a^T dy_i,               dx_i = dx_base_i + A_a^T dv_i,   dA_a = sum_i dv_i x_i^T,  dB_a = s_a sum_i dy_i v_i^T
// The two directions are one kernel with the factors' parts exchanged (down through the factor that is read along the rows of the
// activations, up through the other), then one kernel for the sums over the rows of an adapter.
//
// What bounds them is memory: with rank 16 a value of x takes part in 16 multiply-adds for two bytes.  So no tile of activations goes
// through shared memory: mma.sync does not care which index of the reduction a lane holds as long as both operands agree, so every lane takes
// 16 or 32 consecutive bytes of a row straight into its fragments, each byte once.
//
// Precision.  The tensor cores multiply bf16 exactly and add in fp32.  bf16 tensors enter as they are; an fp32 value enters as the
// sum of bf16 parts: three (24 bits, the value itself) where the result is fp32, so that it has fp32's accuracy, two (16 bits) for the
// low-rank vector of a bf16 result, whose own rounding is 2^-9.  Of the nine products of two values in three parts the three smallest
// are left out: with second parts below 2^-7 and third ones below 2^-15 they are 2^-21 of the product at most, 2^-24 on average.
#include <cooperative_groups.h>

#include "lowrank.cuh"

namespace cg = cooperative_groups;

namespace emoe {
namespace {

constexpr int LR_CLUSTER = 8;      // most CTAs that share a tile
constexpr int LR_IDS_ROWS = 1024;  // most rows whose adapters every CTA looks up by itself

struct LowrankArgs {
  const void *x, *base;  // rows in, rows added to the result (null: zeros)
  const void *down, *up; // forward: A, B; backward: B, A
  const float* scales;   // null: 1
  const int32_t *ids, *off, *perm;
  void* y;               // null: the low-rank vectors alone
  float* v;              // null: not wanted
  int* check_word;
  int32_t *off_out, *perm_out;  // given: one tile more writes the order of the ids there, for the kernels behind
  int n, G, rank, in_dim, out_dim, segments;  // segments: G, or G + 1 with the rows of no adapter as the last
  int skip_none;         // rows of no adapter stay as they are
  size_t x_stride, y_stride;
};

// Which rows this cluster works on: their number and adapter (-1: none) or 0.  Rows are listed in shared memory.  Segments are cut into tiles
// of BT rows, one behind the other.  ids: every CTA counts the rows of each adapter, then lists those of its tile.
template <int BT>
__device__ __forceinline__ int find_rows(const LowrankArgs& a, int tile, int* s_rows, int* s_scan, int* s_count, int* adapter) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int IDS = LR_IDS_ROWS / LR_THREADS;
  int id[IDS];
  if (a.ids) {
#pragma unroll
    for (int i = 0; i < IDS; ++i) {
      const int j = i * LR_THREADS + tid;
      id[i] = j < a.n ? a.ids[j] : -2;
      if (j < a.n && (id[i] < 0 || id[i] >= a.G)) {
        if (id[i] != -1 && tile == 0) atomicOr(a.check_word, CHECK_BAD_EXPERT_ID);
        id[i] = a.G;
      }
    }
    for (int e = tid; e <= a.G; e += LR_THREADS) s_count[e] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < IDS; ++i)
      if (id[i] >= 0) atomicAdd(&s_count[id[i]], 1);
    __syncthreads();
  } else if (tile == 0) {
    check_offsets(a.off, a.segments, a.n, a.check_word);
  }
  // one thread per segment: its tiles, added up
  const auto span = [&](int i) { return a.ids ? RowSpan{0, s_count[i]} : span_of(a.off, i, a.n); };
  RowSpan mine = {0, 0};
  if (tid < a.segments) mine = span(tid);
  const int tiles = (mine.rows + BT - 1) / BT;
  int incl = tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) s_scan[warp] = incl;
  if (tid == 0) s_scan[LR_WARPS] = 0;
  // (a 257th segment, the rows of no adapter beside 256 of them)
  RowSpan last = {0, 0};
  if (a.segments > LR_THREADS) last = span(LR_THREADS);
  __syncthreads();
  int front = 0, all = 0;
  for (int w = 0; w < LR_WARPS; ++w) {
    if (w < warp) front += s_scan[w];
    all += s_scan[w];
  }
  const int first = front + incl - tiles;
  if (tile >= first && tile < first + tiles) {
    s_scan[LR_WARPS] = min(BT, mine.rows - (tile - first) * BT);
    s_scan[LR_WARPS + 1] = mine.begin + (tile - first) * BT;
    s_scan[LR_WARPS + 2] = tid;
  }
  if (tid == 0 && tile >= all && tile < all + (last.rows + BT - 1) / BT) {
    s_scan[LR_WARPS] = min(BT, last.rows - (tile - all) * BT);
    s_scan[LR_WARPS + 1] = last.begin + (tile - all) * BT;
    s_scan[LR_WARPS + 2] = LR_THREADS;
  }
  __syncthreads();
  const int count = s_scan[LR_WARPS], at = s_scan[LR_WARPS + 1], g = s_scan[LR_WARPS + 2];
  if (count == 0) return 0;
  *adapter = g < a.G ? g : -1;
  if (!a.ids) {
    for (int i = tid; i < count; i += LR_THREADS) s_rows[i] = a.perm ? a.perm[at + i] : at + i;
    __syncthreads();
    return count;
  }
  // places at .. at + count - 1 among the rows of the adapter, which a warp's ballots and the counts in front of it give
  unsigned same[IDS];
#pragma unroll
  for (int i = 0; i < IDS; ++i) {
    same[i] = __ballot_sync(0xffffffffu, id[i] == g);
    if (lane == 0) s_count[i * LR_WARPS + warp] = __popc(same[i]);  // (every thread has its counts: they are read in front of the last barrier)
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < IDS; ++i) {
    if (id[i] != g) continue;
    int place = __popc(same[i] & ((1u << lane) - 1u));
    for (int c = 0; c < i * LR_WARPS + warp; ++c) place += s_count[c];
    if (place >= at && place < at + count) s_rows[place - at] = i * LR_THREADS + tid;
  }
  __syncthreads();
  return count;
}

// The order of at most LR_IDS_ROWS ids as launch_sort_pairs writes it (ids of no adapter behind the others), by one CTA beside those that multiply: a
// launch in front of them takes some 4 us (backward, bf16, 64 rows of 8 adapters, 2048 -> 2048, 16.0/12.2; 1000 of 60, 512 -> 512, 19.8/14.9).  A warp owns consecutive rows: it counts them by adapter, then hands out their places.
__device__ __forceinline__ void write_order(const LowrankArgs& a, int (*first)[EMOE_MAX_EXPERTS + 1], int* s_scan) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, segments = a.G + 1, bits = 32 - __clz(a.G);
  constexpr int STEPS = LR_IDS_ROWS / LR_THREADS;
  for (int i = tid; i < LR_WARPS * segments; i += LR_THREADS) first[i / segments][i % segments] = 0;
  __syncthreads();
  int id[STEPS], front[STEPS];
  unsigned same[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int row = (warp * STEPS + i) * 32 + lane;
    id[i] = row < a.n ? a.ids[row] : -2;
    if (row < a.n && (id[i] < 0 || id[i] >= a.G)) id[i] = a.G;
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    same[i] = __ballot_sync(0xffffffffu, id[i] >= 0);
    for (int b = 0; b < bits; ++b) {
      const unsigned set = __ballot_sync(0xffffffffu, id[i] >> b & 1);
      same[i] &= (id[i] >> b & 1) ? set : ~set;
    }
    front[i] = __popc(same[i] & ((1u << lane) - 1u));
    if (id[i] >= 0 && front[i] == 0) first[warp][id[i]] += __popc(same[i]);
    __syncwarp();
  }
  __syncthreads();
  const auto rows_of = [&](int e) {
    int sum = 0;
    for (int w = 0; w < LR_WARPS; ++w) sum += first[w][e];
    return sum;
  };
  const int rows = tid < segments ? rows_of(tid) : 0;
  int incl = rows;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  int before = incl - rows, all = 0;
  for (int w = 0; w < LR_WARPS; ++w) {
    if (w < warp) before += s_scan[w];
    all += s_scan[w];
  }
  const auto hand_out = [&](int e, int at) {
    a.off_out[e] = at;
    for (int w = 0; w < LR_WARPS; ++w) {
      const int c = first[w][e];
      first[w][e] = at;
      at += c;
    }
  };
  if (tid < segments) hand_out(tid, before);
  if (tid == 0) {
    if (segments > LR_THREADS) hand_out(LR_THREADS, all);  // a 257th segment
    a.off_out[segments] = a.n;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    if (id[i] >= 0) a.perm_out[first[warp][id[i]] + front[i]] = (warp * STEPS + i) * 32 + lane;
    __syncwarp();
    if (id[i] >= 0 && front[i] == 0) first[warp][id[i]] += __popc(same[i]);
    __syncwarp();
  }
}

// RT: rank in tiles of 16; NT: rows in tiles of 8; BACK: the down factor is B ([reduction][rank]), the up factor A ([rank][out]).
template <typename T, int RT, int NT, bool BACK>
struct Lowrank {
  static constexpr int BT = NT * 8, MT = (NT + 1) / 2, RP = RT * 16;
  static constexpr int PI = Parts<T>::IN, PV = Parts<T>::VEC;
  static constexpr int WORDS = RT * NT >= 16 || (sizeof(T) == 4 && RT * NT >= 8) ? 4 : 8;  // of a row per lane and step: 16 or 32 bytes
  static constexpr int VALS = WORDS * 4 / static_cast<int>(sizeof(T)), STEP = VALS * 4, KS = VALS / 4;
  static constexpr int V_STRIDE = 16 * (RT == 1 ? 1 : RT == 2 ? 3 : 5);  // bf16 values: an odd number of 32-byte pieces, no bank met twice
  static constexpr int RED_FLOATS = LR_WARPS / 2 * RT * NT * 4 * 32, PART_FLOATS = BT * RP;
  static constexpr size_t SMEM = sizeof(float) * (RED_FLOATS + PART_FLOATS) + 2ull * PV * MT * 16 * V_STRIDE;

  // rank index of row g (half 0) or g + 8 (half 1) of tile m of the down factor's fragments
  __device__ static __forceinline__ int rank_of(int m, int g, int half) { return BACK ? 2 * RT * g + 2 * m + half : 16 * m + g + 8 * half; }
  // place of a rank index in the low-rank vectors: the four that lane q of step s multiplies with lie together
  __device__ static __forceinline__ int place_of(int r) { return r % (4 * RT) / 4 * 16 + r / (4 * RT) * 4 + r % 4; }

  // N values of a factor's row from `first` on, those at or beyond `end` zero
  template <int N>
  __device__ static __forceinline__ void load_factor(const T* row, int first, int end, bool whole, uint32_t (&w)[N * sizeof(T) / 4]) {
    constexpr int WN = N * sizeof(T) / 4;
#pragma unroll
    for (int i = 0; i < WN; ++i) w[i] = 0;
    if (whole) {
      if (first < end) {
        if constexpr (WN == 1) w[0] = *reinterpret_cast<const uint32_t*>(row + first);
        else if constexpr (WN == 2) {
          const uint2 u = *reinterpret_cast<const uint2*>(row + first);
          w[0] = u.x; w[1] = u.y;
        } else {
#pragma unroll
          for (int i = 0; i < WN; i += 4)
            if (first + i * 4 / static_cast<int>(sizeof(T)) < end) {
              const uint4 u = load16_keep(reinterpret_cast<const char*>(row + first) + 4 * i);
              w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
            }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (first + i < end) {
          if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(row)[first + i];
          else w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[first + i]) << (16 * (i % 2));
        }
    }
  }
};

template <typename T, int RT, int NT, bool BACK>
__global__ void __launch_bounds__(LR_THREADS, NT == 1 || RT <= (sizeof(T) == 2 ? 2 : 1) ? 2 : 1) lowrank_kernel(LowrankArgs a) {
  using L = Lowrank<T, RT, NT, BACK>;
  constexpr int BT = L::BT, RP = L::RP, PI = L::PI, PV = L::PV, WORDS = L::WORDS, KS = L::KS;
  extern __shared__ __align__(16) char smem[];
  float* s_red = reinterpret_cast<float*>(smem);
  float* s_part = s_red + L::RED_FLOATS;
  __nv_bfloat16* s_v = reinterpret_cast<__nv_bfloat16*>(s_part + L::PART_FLOATS);
  __shared__ int s_rows[BT], s_scan[LR_WARPS + 3], s_count[EMOE_MAX_EXPERTS + 1];
  static_assert(LR_IDS_ROWS / 32 <= EMOE_MAX_EXPERTS, "the warps' counts lie where the adapters' were");
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  const int ctas = static_cast<int>(cluster.num_blocks()), cta = static_cast<int>(cluster.block_rank());
  pdl_wait();
  pdl_trigger();
  if constexpr (BACK) {
    __shared__ int first[LR_WARPS][EMOE_MAX_EXPERTS + 1];
    if (a.perm_out && blockIdx.x / ctas == gridDim.x / ctas - 1) {
      if (cta == 0) write_order(a, first, s_scan);
      return;
    }
  }
  int adapter = -1;
  const int count = find_rows<BT>(a, blockIdx.x / ctas, s_rows, s_scan, s_count, &adapter);
  if (count == 0 || (adapter < 0 && a.skip_none && !a.v)) return;  // the whole cluster
  const T* down = static_cast<const T*>(a.down) + static_cast<size_t>(adapter < 0 ? 0 : adapter) * a.rank * a.in_dim;
  const T* up = static_cast<const T*>(a.up) + static_cast<size_t>(adapter < 0 ? 0 : adapter) * a.rank * a.out_dim;

  // ---- down: v = A x (forward), B^T dy (backward); every warp of the cluster takes a share of the reduction
  if (adapter >= 0) {
    float acc[RT][NT][4] = {};
    const T* row[NT];
    bool live[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      live[t] = t * 8 + g < count;
      row[t] = static_cast<const T*>(a.x) + static_cast<size_t>(live[t] ? s_rows[t * 8 + g] : 0) * a.x_stride;
    }
    const bool whole = a.rank % (2 * RT) == 0;  // (backward) a lane's run of ranks is one aligned word of each row
    const int steps = (a.in_dim + L::STEP - 1) / L::STEP;
    for (int step = cta * LR_WARPS + warp; step < steps; step += ctas * LR_WARPS) {
      const int k = step * L::STEP + q * L::VALS;  // this lane's first index of the reduction
      uint32_t xw[NT][WORDS];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
          uint4 u = make_uint4(0, 0, 0, 0);
          const int at = k + i * 4 / static_cast<int>(sizeof(T));
          if (live[t] && at < a.in_dim) u = load16(row[t] + at);
          xw[t][i] = u.x; xw[t][i + 1] = u.y; xw[t][i + 2] = u.z; xw[t][i + 3] = u.w;
        }
      uint32_t fw[BACK ? 1 : RT][2][BACK ? 1 : WORDS];
      if constexpr (!BACK) {
#pragma unroll
        for (int m = 0; m < RT; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = L::rank_of(m, g, h);
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
              uint4 u = make_uint4(0, 0, 0, 0);
              const int at = k + i * 4 / static_cast<int>(sizeof(T));
              if (r < a.rank && at < a.in_dim) u = load16_keep(down + static_cast<size_t>(r) * a.in_dim + at);
              fw[m][h][i] = u.x; fw[m][h][i + 1] = u.y; fw[m][h][i + 2] = u.z; fw[m][h][i + 3] = u.w;
            }
          }
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        uint32_t af[RT][PI][4];
        if constexpr (!BACK) {
#pragma unroll
          for (int m = 0; m < RT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if constexpr (sizeof(T) == 2) {
                af[m][0][h] = fw[m][h][2 * s];
                af[m][0][2 + h] = fw[m][h][2 * s + 1];
              } else {
                uint32_t p[PI];
                split_pair<PI>(__uint_as_float(fw[m][h][4 * s]), __uint_as_float(fw[m][h][4 * s + 1]), p);
#pragma unroll
                for (int i = 0; i < PI; ++i) af[m][i][h] = p[i];
                split_pair<PI>(__uint_as_float(fw[m][h][4 * s + 2]), __uint_as_float(fw[m][h][4 * s + 3]), p);
#pragma unroll
                for (int i = 0; i < PI; ++i) af[m][i][2 + h] = p[i];
              }
            }
        } else {
          // four rows of B, of each the ranks 2 RT g ..: pairs of rows are interleaved into fragments
          constexpr int WN = 2 * RT * static_cast<int>(sizeof(T)) / 4;
          uint32_t w[4][WN];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = k + 4 * s + i;
            L::template load_factor<2 * RT>(down + static_cast<size_t>(at) * a.rank, 2 * RT * g, at < a.in_dim ? a.rank : 0, whole, w[i]);
          }
#pragma unroll
          for (int m = 0; m < RT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int half = 0; half < 2; ++half) {  // rows 0 and 1, rows 2 and 3
                if constexpr (sizeof(T) == 2) {
                  af[m][0][2 * half + h] = __byte_perm(w[2 * half][m], w[2 * half + 1][m], h ? 0x7632 : 0x5410);
                } else {
                  uint32_t p[PI];
                  split_pair<PI>(__uint_as_float(w[2 * half][2 * m + h]), __uint_as_float(w[2 * half + 1][2 * m + h]), p);
#pragma unroll
                  for (int i = 0; i < PI; ++i) af[m][i][2 * half + h] = p[i];
                }
              }
        }
        uint32_t bf[NT][PI][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if constexpr (sizeof(T) == 2) {
            bf[t][0][0] = xw[t][2 * s];
            bf[t][0][1] = xw[t][2 * s + 1];
          } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t p[PI];
              split_pair<PI>(__uint_as_float(xw[t][4 * s + 2 * half]), __uint_as_float(xw[t][4 * s + 2 * half + 1]), p);
#pragma unroll
              for (int i = 0; i < PI; ++i) bf[t][i][half] = p[i];
            }
          }
        }
#pragma unroll
        for (int m = 0; m < RT; ++m) {
          const uint32_t(&am)[1][PI][4] = reinterpret_cast<const uint32_t(&)[1][PI][4]>(af[m]);
          if constexpr (PI == 1) {
            mma_parts_of<false>(acc[m], am, bf);
          } else {  // the tensor cores cut what they add: sixteen products of fp32 values are summed by themselves, then added with rounding
            float d[NT][4];
            mma_parts_of<true>(d, am, bf);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[m][t][i] += d[t][i];
          }
        }
      }
    }
    // the warps' shares, added pairwise in a fixed order
#pragma unroll
    for (int half = LR_WARPS / 2; half >= 1; half >>= 1) {
      float* slot = s_red + (warp & (half - 1)) * (RT * NT * 4 * 32) + lane;
      if (warp >= half && warp < 2 * half) {
#pragma unroll
        for (int i = 0; i < RT * NT * 4; ++i) slot[i * 32] = (&acc[0][0][0])[i];
      }
      __syncthreads();
      if (warp < half) {
#pragma unroll
        for (int i = 0; i < RT * NT * 4; ++i) (&acc[0][0][0])[i] += slot[i * 32];
      }
      __syncthreads();
    }
    if (warp == 0) {
#pragma unroll
      for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s_part[(t * 8 + 2 * q + i % 2) * RP + L::rank_of(m, g, i / 2)] = acc[m][t][i];
    }
  }
  if (ctas > 1) cluster.sync();
  else __syncthreads();

  // ---- the vectors whole, scaled, in bf16 parts
  const float scale = a.scales && adapter >= 0 ? a.scales[adapter] : 1.f;
  for (int i = tid; i < L::MT * 16 * RP; i += LR_THREADS) {
    const int t = i / RP, r = i % RP;
    float v = 0.f;
    if (t < BT && adapter >= 0 && r < a.rank) {  // (beyond the rank an infinite activation has met zeros)
      float part[LR_CLUSTER];  // asked for together: a load from another SM takes long
#pragma unroll
      for (int c = 0; c < LR_CLUSTER; ++c) part[c] = c < ctas ? cluster.map_shared_rank(s_part, c)[t * RP + r] : 0.f;
#pragma unroll
      for (int c = 0; c < LR_CLUSTER; ++c) v += part[c];
    }
    const float scaled = scale * v;
    if (a.v && t < count && r < a.rank && t % ctas == cta) a.v[static_cast<size_t>(s_rows[t]) * a.rank + r] = BACK ? scaled : v;
    uint32_t p[PV];
    split_pair<PV>(scaled, 0.f, p);
#pragma unroll
    for (int j = 0; j < PV; ++j)
      s_v[(j * L::MT * 16 + t) * L::V_STRIDE + L::place_of(r)] = __ushort_as_bfloat16(static_cast<unsigned short>(p[j] & 0xffffu));
  }
  if (ctas > 1) cluster.sync();  // nobody leaves while another CTA reads its share
  else __syncthreads();
  if (!a.y || (adapter < 0 && a.skip_none)) return;

  // ---- up: y = base + B v; a warp takes 32 channels of all rows at a time, a lane eight neighbouring ones of two rows
  const bool whole = a.rank % (RT == 1 ? 4 : 8) == 0;  // (forward) a lane's run of ranks is whole aligned words
  const int groups = (a.out_dim + 31) / 32;
  for (int group = cta * LR_WARPS + warp; group < groups; group += ctas * LR_WARPS) {
    const int n0 = group * 32, mine = n0 + 8 * q;  // the lane's channels of the result
    uint32_t bw[L::MT][2][sizeof(T) * 2];
#pragma unroll
    for (int t = 0; t < L::MT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = t * 16 + h * 8 + g;
#pragma unroll
        for (int w = 0; w < static_cast<int>(sizeof(T)) * 2; w += 4) {
          uint4 u = make_uint4(0, 0, 0, 0);
          if (a.base && i < count && mine < a.out_dim)
            u = load16(static_cast<const T*>(a.base) + static_cast<size_t>(s_rows[i]) * a.y_stride + mine + w * 4 / static_cast<int>(sizeof(T)));
          bw[t][h][w] = u.x; bw[t][h][w + 1] = u.y; bw[t][h][w + 2] = u.z; bw[t][h][w + 3] = u.w;
        }
      }
    // up factor: tile i of eight columns holds the channels 8 c' + 2 i + (c & 1), c = 2 c' + (c & 1) the column of this lane
    uint32_t uf[RT][4][PI][2];
    if constexpr (!BACK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = n0 + 8 * (g >> 1) + 2 * i + (g & 1);
        constexpr int WN = 4 * RT * static_cast<int>(sizeof(T)) / 4;
        uint32_t w[WN];
        L::template load_factor<4 * RT>(up + static_cast<size_t>(ch) * a.rank, 4 * RT * q, ch < a.out_dim && adapter >= 0 ? a.rank : 0, whole, w);
#pragma unroll
        for (int s = 0; s < RT; ++s) {
          if constexpr (sizeof(T) == 2) {
            uf[s][i][0][0] = w[2 * s];
            uf[s][i][0][1] = w[2 * s + 1];
          } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t p[PI];
              split_pair<PI>(__uint_as_float(w[4 * s + 2 * half]), __uint_as_float(w[4 * s + 2 * half + 1]), p);
#pragma unroll
              for (int j = 0; j < PI; ++j) uf[s][i][j][half] = p[j];
            }
          }
        }
      }
    } else {
      const int ch = n0 + 8 * (g >> 1);
#pragma unroll
      for (int s = 0; s < RT; ++s)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t w[2][sizeof(T) * 2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = 4 * RT * q + 4 * s + 2 * half + j;
            L::template load_factor<8>(up + static_cast<size_t>(r) * a.out_dim, ch, r < a.rank && adapter >= 0 ? a.out_dim : 0, true, w[j]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2) {
              uf[s][i][0][half] = __byte_perm(w[0][i], w[1][i], (g & 1) ? 0x7632 : 0x5410);
            } else {
              uint32_t p[PI];
              const bool odd = g & 1;
              split_pair<PI>(__uint_as_float(odd ? w[0][2 * i + 1] : w[0][2 * i]), __uint_as_float(odd ? w[1][2 * i + 1] : w[1][2 * i]), p);
#pragma unroll
              for (int j = 0; j < PI; ++j) uf[s][i][j][half] = p[j];
            }
          }
        }
    }
#pragma unroll
    for (int t = 0; t < L::MT; ++t) {
      float d[4][4] = {};
#pragma unroll
      for (int s = 0; s < RT; ++s) {
        uint32_t vf[1][PV][4];
#pragma unroll
        for (int j = 0; j < PV; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint2 u = *reinterpret_cast<const uint2*>(s_v + (j * L::MT * 16 + t * 16 + h * 8 + g) * L::V_STRIDE + s * 16 + 4 * q);
            vf[0][j][h] = u.x;
            vf[0][j][2 + h] = u.y;
          }
        mma_parts_of<false>(d, vf, uf[s]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = t * 16 + h * 8 + g;
        if (i >= count || mine >= a.out_dim) continue;
        Piece<T, 8> p;
#pragma unroll
        for (int w = 0; w < Piece<T, 8>::WORDS; ++w) p.w[w] = bw[t][h][w];
        float f[8];
        widen<T, 8>(p, f);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          f[2 * c] += d[c][2 * h];
          f[2 * c + 1] += d[c][2 * h + 1];
        }
        store_piece<T, 8>(static_cast<T*>(a.y) + static_cast<size_t>(s_rows[i]) * a.y_stride + mine, narrow<T, 8>(f));
      }
    }
  }
}

// ---- gradients of the factors -------------------------------------------------------------------

// out[c][r] = sum over an adapter's rows of act[row][c] vec[row][r]:  dB from dy and s v (out [N][rank]), dA from x and dv (out [rank][K]).
// The reduction runs over rows, so a lane takes the same eight channels of four rows and interleaves pairs of rows.  A CTA owns an even
// run of the rows and 32 channels per warp; the vectors of 64 rows at a time lie in shared memory as pairs of rows in three bf16
// parts.  A segment that is one run's alone is written at once, else the runs' shares are joined behind this kernel, in order.
// Two tiles of 16 channels per warp leave two CTAs an SM; with four a CTA has one for itself and, beyond rank 16, too few registers (us, whole
// call, fp32, four / two: 1561 x 4864 -> 3360, rank 16 75/72; 6000 x 1024 -> 1024, rank 32 110/95; 2048 x 2048 -> 2048, rank 64 158/145).
constexpr int GR_ROWS = 64, GR_TILES = 2, GR_CHANNELS = GR_TILES * 16 * LR_WARPS, GR_CTAS = 2;
constexpr int LR_MAX_DIM = 65535 / 2 * GR_CHANNELS;  // the blocks of dB and dA stand side by side in one grid, 65535 high at most

struct GradArgs {
  const void* act[2];     // dy, x
  const float* vec[2];    // v, dv
  size_t stride[2];
  int dim[2];             // out_dim, in_dim
  float* out[2];          // dB, dA (null: not wanted)
  const float* scales;    // of dB
  const int32_t *off, *perm;
  float* part[2];         // [2 x runs][dim][rank]: shares of segments that several runs have
  int* check_word;
  int n, G, rank, runs[2], blocks[2];
};

template <typename T, int RT>
__global__ void __launch_bounds__(LR_THREADS, GR_CTAS) lowrank_grad_kernel(GradArgs a) {
  constexpr int MT = GR_TILES, CH = 2 * MT, WORDS = CH * static_cast<int>(sizeof(T)) / 4, NR = RT * 2, RP = RT * 16, PI = Parts<T>::IN, PAIRS = GR_ROWS / 2, W_STRIDE = RP + 4;
  __shared__ uint32_t s_vec[3][PAIRS][W_STRIDE];
  __shared__ int s_rows[GR_ROWS];
  __shared__ TileList list;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  pdl_wait();
  pdl_trigger();
  const int which = static_cast<int>(blockIdx.y) >= a.blocks[0], block = blockIdx.y - (which ? a.blocks[0] : 0);
  if (static_cast<int>(blockIdx.x) >= a.runs[which]) return;
  const TileRun run = list_tiles<GR_ROWS>(list, a.off, a.G, a.n, blockIdx.x, a.runs[which]);
  if (run.lo >= run.hi) return;
  const int dim = a.dim[which], c0 = block * GR_CHANNELS + (warp * 8 + g) * CH;  // this lane's channels
  const T* act = static_cast<const T*>(a.act[which]);
  const float* vec = a.vec[which];
  float acc[MT][NR][4] = {};
  for (RunWalk<GR_ROWS> walk(list, run); walk.more();) {
    const Tile tile = walk.next();
    const int rows = tile.rows, segment = walk.segment;
    const float scale = which == 0 && a.scales ? a.scales[segment] : 1.f;
    __syncthreads();  // the vectors of the rows before have been used
    for (int i = tid; i < GR_ROWS; i += LR_THREADS) s_rows[i] = i < rows ? (a.perm ? a.perm[tile.begin + i] : tile.begin + i) : -1;
    __syncthreads();
    for (int i = tid; i < PAIRS * RP; i += LR_THREADS) {
      const int pair = i / RP, r = i % RP, ra = s_rows[2 * pair], rb = s_rows[2 * pair + 1];
      const float va = ra >= 0 && r < a.rank ? scale * vec[static_cast<size_t>(ra) * a.rank + r] : 0.f;
      const float vb = rb >= 0 && r < a.rank ? scale * vec[static_cast<size_t>(rb) * a.rank + r] : 0.f;
      uint32_t p[3];
      split_pair<3>(va, vb, p);
#pragma unroll
      for (int j = 0; j < 3; ++j) s_vec[j][pair][r] = p[j];
    }
    __syncthreads();
#pragma unroll (RT == 1 ? 2 : 1)
    for (int k = 0; k < GR_ROWS; k += 16) {
      if (k >= rows) break;
      uint32_t w[4][WORDS];  // this lane's channels of rows 4 q .. 4 q + 3
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = s_rows[k + 4 * q + i];
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[i][j] = 0;
        if (row >= 0 && c0 < dim) load_words(act + static_cast<size_t>(row) * a.stride[which] + c0, w[i]);
      }
      uint32_t af[MT][PI][4];  // tile m: channels c0 + 2 m (rows g) and c0 + 2 m + 1 (rows g + 8)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if constexpr (sizeof(T) == 2) {
              af[m][0][2 * half + h] = __byte_perm(w[2 * half][m], w[2 * half + 1][m], h ? 0x7632 : 0x5410);
            } else {
              uint32_t p[PI];
              split_pair<PI>(__uint_as_float(w[2 * half][2 * m + h]), __uint_as_float(w[2 * half + 1][2 * m + h]), p);
#pragma unroll
              for (int j = 0; j < PI; ++j) af[m][j][2 * half + h] = p[j];
            }
          }
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        uint32_t bf[1][3][2];
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) bf[0][j][half] = s_vec[j][k / 2 + 2 * q + half][nr * 8 + g];
        // the tensor cores cut what they add: sixteen rows are summed by themselves, then added with rounding
        float d[MT][4];
        mma_parts_of<true>(d, af, bf);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][nr][i] += d[m][i];
      }
    }
    if (!tile.ends) continue;
    const size_t size = static_cast<size_t>(dim) * a.rank;
    const int share = share_of(list, run, segment, blockIdx.x);
    float* out = share < 0 ? a.out[which] + segment * size : a.part[which] + share * size;
    // c0 + 2 m + h, rank nr * 8 + 2 q + b
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int r = nr * 8 + 2 * q + b;
        if (r >= a.rank || c0 >= dim) continue;
        if (which == 0) {
#pragma unroll
          for (int c = 0; c < CH; ++c) out[static_cast<size_t>(c0 + c) * a.rank + r] = acc[c / 2][nr][2 * (c % 2) + b];
        } else {
          float4* o = reinterpret_cast<float4*>(out + static_cast<size_t>(r) * dim + c0);
#pragma unroll
          for (int m = 0; m < MT; m += 2) o[m / 2] = make_float4(acc[m][nr][b], acc[m][nr][2 + b], acc[m + 1][nr][b], acc[m + 1][nr][2 + b]);
        }
      }
#pragma unroll
    for (int i = 0; i < MT * NR * 4; ++i) (&acc[0][0][0])[i] = 0.f;
  }
}

// Joins the shares of segments that several runs have, in order, and clears the gradients of adapters without rows.  grid: (adapters,
// pieces of a gradient, dB and dA); H: rows of a tile of the kernel in front; CHECK: no kernel in front has looked at the offsets.
template <int H, bool CHECK>
__global__ void __launch_bounds__(LR_THREADS) lowrank_join_kernel(GradArgs a) {
  __shared__ TileList list;
  const int tid = threadIdx.x, adapter = blockIdx.x, which = blockIdx.z;
  // (the offsets are older than the kernel in front, which waited before its trigger)
  const TileRun run = list_tiles<H>(list, a.off, a.G, a.n, 0, a.runs[which]);
  pdl_wait();
  pdl_trigger();
  if (CHECK && blockIdx.x == 0 && blockIdx.y == 0 && which == 0) check_offsets(a.off, a.G, a.n, a.check_word);
  if (!a.out[which]) return;
  const int first = list.first[adapter], end = list.first[adapter + 1], c0 = first / run.per, c1 = end > first ? (end - 1) / run.per : c0 - 1;
  if (c0 == c1) return;
  const size_t words = static_cast<size_t>(a.dim[which]) * a.rank / 4;  // dim is a multiple of 8
  float4* out = reinterpret_cast<float4*>(a.out[which]) + adapter * words;
  const float4* in = reinterpret_cast<const float4*>(a.part[which]);
  for (size_t i = static_cast<size_t>(blockIdx.y) * LR_THREADS + tid; i < words; i += static_cast<size_t>(gridDim.y) * LR_THREADS) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
      const float4 u = in[(2 * c + (c < c1)) * words + i];
      s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
    }
    out[i] = s;
  }
}

// ---- launches -----------------------------------------------------------------------------------

struct LowrankLayout {
  size_t off, perm, vec, planes, part[2], total;  // vec: dv, or the vectors in the order; planes: their shares
  int runs[2];                                    // of the outer products: dB, dA
};

int blocks_of(int dim, int channels) { return (dim + channels - 1) / channels; }
// Even runs of the rows, for `blocks` CTAs per run where the GPU holds `slots` at once: as many as run side by side, or whole multiples
// of that where a run would be longer than `most` tiles.
int runs_for(int n, int segments, int blocks, int slots, int tile, int most) {
  const int side = slots / blocks > 0 ? slots / blocks : 1, tiles = (n + tile - 1) / tile + (segments < n ? segments : n);
  const int least = (tiles + most - 1) / most, runs = (least + side - 1) / side * side;
  return runs < tiles ? runs : tiles;
}
// Which bf16 calls take the streaming kernels, by the bytes of the rows read and written: they (and their launches) cost some 10 us more at the
// start and gain from there on.  The fused kernel's time goes in steps, by rounds of clusters, so that near the limits either may be the faster one, by a
// fifth at most.  us, fused / streaming, 8 adapters with ids (in brackets 16 by offsets):
//   forward, 4096 -> 4096   rank 16: 2048 rows 22/32 (27/24), 3200 rows 35/33 (29/26), 4557 rows 35/40 (40/34), 6000 rows 49/43 (44/36),
//                           8192 rows 55/53 (49/45); rank 32: 4557 rows 38/44 (49/38); rank 64: 1024 rows 24/34 (24/26),
//                           1300 rows (33/28), 1536 rows 38/33 (34/29)
//           2048 -> 2048    rank 16: 9114 rows 35/39 (28/32), 12000 rows 51/44;  4096 -> 14336, rank 32: 2000 rows (42/45), 4099 rows (74/66)
//   backward, 4096 -> 4096  rank 16: 512 rows 28/29 (24/26), 1100 rows 45/38 (1024: 40/29); rank 64: 256 rows (48/48), 384 rows 44/38 (51/49)
//           1024 -> 1024    rank 16: 2048 rows 27/31 (23/23), 4096 rows (27/27);  2048 -> 2048: 1342 rows 32/31 (24/25)
bool takes_stream(const emoe_lowrank_desc& D, int n, bool back) {
  const double K = D.in_dim, N = D.out_dim, bytes = 2.0 * n * (back ? 3 * K + N : K + 2 * N);
  return D.dtype == EMOE_DTYPE_BF16 && bytes > (back ? (D.rank > 32 ? 12e6 : 20e6) : (D.rank > 32 ? 32e6 : 80e6));
}

LowrankLayout lowrank_layout(const emoe_lowrank_desc& D, int n, bool back) {
  const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  const bool stream = takes_stream(D, n, back);
  LowrankLayout w{};
  const size_t vectors = sizeof(float) * static_cast<size_t>(n) * D.rank;
  size_t o = 0;
  w.off = o;  o += up(sizeof(int32_t) * (D.n_adapters + 2));
  w.perm = o; o += up(sizeof(int32_t) * static_cast<size_t>(n));
  w.vec = o;  o += up(vectors);
  w.planes = o;
  if (stream) o += up(vectors * blocks_of(D.in_dim > D.out_dim ? D.in_dim : D.out_dim, stream_channels(D.rank)));
  for (int i = 0; i < 2; ++i) {
    const size_t dim = i ? D.in_dim : D.out_dim;
    w.part[i] = o;
    if (!back) continue;
    // 1024 rows at most per run, as accuracy goes on the streaming path
    if (stream) w.runs[i] = runs_for(n, D.n_adapters, blocks_of(static_cast<int>(dim), stream_channels(D.rank)), GPU_SMS, STREAM_ROWS, STREAM_RUN);
    else  // (both outer products are one launch)
      w.runs[i] = runs_for(n, D.n_adapters, blocks_of(D.in_dim, GR_CHANNELS) + blocks_of(D.out_dim, GR_CHANNELS),
                           GR_CTAS * GPU_SMS, GR_ROWS, STREAM_RUN * STREAM_ROWS / GR_ROWS);
    // Two shares per run.  What is reserved grows with n, dim and rank alike, so that a context that is made for the largest call serves all:
    // runs <= slots / blocks + tiles / 8 + 1 and slots / blocks * dim <= slots * 512; runs <= tiles.
    const size_t tiles = (static_cast<size_t>(n) + GR_ROWS - 1) / GR_ROWS + (D.n_adapters < n ? D.n_adapters : n);
    const size_t even = static_cast<size_t>(2 * GPU_SMS) * 512 + (tiles / STREAM_RUN + 2) * dim;
    o += up(sizeof(float) * 2 * (tiles * dim < even ? tiles * dim : even) * D.rank);
  }
  w.total = o;
  return w;
}

template <typename T, int RT, int NT, bool BACK>
cudaError_t launch_tile(const LowrankArgs& a, int tiles, int ctas, cudaStream_t st) {
  using L = Lowrank<T, RT, NT, BACK>;
  if (L::SMEM > 40 * 1024) {
    const cudaError_t e = allow_smem<lowrank_kernel<T, RT, NT, BACK>>(static_cast<int>(L::SMEM));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles) * ctas);
  cfg.blockDim = dim3(LR_THREADS);
  cfg.dynamicSmemBytes = L::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {static_cast<unsigned>(ctas), 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl_enabled ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, lowrank_kernel<T, RT, NT, BACK>, a);
}

// Clusters of 1, 2, 4 and 8 CTAs that the GPU holds at once, of kernels with one, two and three CTAs per SM (larger ones leave SMs of a
// part of the GPU empty).
constexpr int CLUSTERS_HELD[3][4] = {{148, 74, 33, 15}, {296, 148, 71, 33}, {444, 222, 104, 48}};

template <typename T, bool BACK>
cudaError_t launch_lowrank(const LowrankArgs& a, cudaStream_t st) {
  // Rows per tile, 8 or 32, and CTAs per tile: what takes least time as rounds of clusters x (1 + 0.15 per doubling of the cluster + what a CTA
  // multiplies), with 32 rows at the price of eight where the registers leave their kernel an SM for itself, of twice eight where it shares one.  Over 124 measured
  // calls (both directions and types, rank 8 to 64, 100 to 4000 rows of 2 to 64 adapters) that is 1.3 % from the fastest choice on average, 19 % at
  // worst.  us, forward, 1024 rows, 2048 -> 2048, four adapters: fp32, rank 32, eight rows x 1 / 2 / 4 CTAs 26.9/21.6/26.9, 32 rows x 1 / 2
  // / 4 48.5/29.3/31.5; rank 16 21.1/16.1/21.1, 31.6/20.3/15.8.  64 rows were slower or as fast everywhere.
  const int segments = a.segments < a.n ? a.segments : a.n;
  const int rt = a.rank <= 16 ? 1 : a.rank <= 32 ? 2 : 4;
  const int held[2] = {sizeof(T) == 2 && rt == 1 && !BACK ? 3 : 2, rt <= (sizeof(T) == 2 ? 2 : 1) ? 2 : 1};  // CTAs per SM
  const double share = (static_cast<double>(a.in_dim) + a.out_dim) / 2048;
  double least = 0.;
  int nt = 1, ctas = 1;
  for (int i = 0; i < 2; ++i)
    for (int log = 0; log < 4; ++log) {
      const int rows = i ? 32 : 8, mean_tiles = a.n / rows + (segments + 1) / 2, at_once = CLUSTERS_HELD[held[i] - 1][log];
      const double cost = ((mean_tiles + at_once - 1) / at_once) * (1. + 0.15 * log + (i ? held[1] : 1) * share / (1 << log));
      if ((i == 0 && log == 0) || cost < least) {
        least = cost;
        nt = rows / 8;
        ctas = 1 << log;
      }
    }
  const int tiles = a.n / (nt * 8) + segments + (a.perm_out ? 1 : 0);
  const auto by_rows = [&](auto ranks) -> cudaError_t {
    constexpr int RT = decltype(ranks)::value;
    return nt == 1 ? launch_tile<T, RT, 1, BACK>(a, tiles, ctas, st) : launch_tile<T, RT, 4, BACK>(a, tiles, ctas, st);
  };
  if (rt == 1) return by_rows(std::integral_constant<int, 1>());
  if (rt == 2) return by_rows(std::integral_constant<int, 2>());
  return by_rows(std::integral_constant<int, 4>());
}

cudaError_t launch_join(const GradArgs& a, bool stream, bool check, cudaStream_t st) {
  const size_t dim = a.dim[0] > a.dim[1] ? a.dim[0] : a.dim[1], shares = (dim * a.rank / 4 + LR_THREADS - 1) / LR_THREADS;
  // CTAs of an adapter's gradient: few adapters share all SMs (8192 x 4096 -> 4096, one adapter, whole call 77/71 us)
  const size_t most = 2 * GPU_SMS / a.G > 32 ? 2 * GPU_SMS / a.G : 32;
  const dim3 grid(a.G, static_cast<unsigned>(shares < most ? shares : most), 2);
  const auto go = [&](auto kernel) { return launch_chain(kernel, grid, dim3(LR_THREADS), 0, st, a); };
  if (check) return stream ? go(lowrank_join_kernel<STREAM_ROWS, true>) : go(lowrank_join_kernel<GR_ROWS, true>);
  return stream ? go(lowrank_join_kernel<STREAM_ROWS, false>) : go(lowrank_join_kernel<GR_ROWS, false>);
}

template <typename T>
cudaError_t launch_grads(const GradArgs& a, cudaStream_t st) {
  const dim3 grid(a.runs[0] > a.runs[1] ? a.runs[0] : a.runs[1], a.blocks[0] + a.blocks[1]);
  if (a.rank <= 16) return launch_chain(lowrank_grad_kernel<T, 1>, grid, dim3(LR_THREADS), 0, st, a);
  if (a.rank <= 32) return launch_chain(lowrank_grad_kernel<T, 2>, grid, dim3(LR_THREADS), 0, st, a);
  return launch_chain(lowrank_grad_kernel<T, 4>, grid, dim3(LR_THREADS), 0, st, a);
}

// Many bf16 rows: rows that go down and, backward, the outer products; the vectors' sum; rows that come up.
cudaError_t launch_many(const LowrankArgs& a, bool back, const GradArgs* ga, char* ws, const LowrankLayout& w, cudaStream_t st) {
  using bf16 = __nv_bfloat16;
  float *vec = reinterpret_cast<float*>(ws + w.vec), *planes = reinterpret_cast<float*>(ws + w.planes);
  const bool vectors = a.y || a.v || (back && ga->out[1]);
  const auto outer = [&](int which, StreamArgs* s) {
    s->vec = which ? vec : ga->vec[0];
    s->vec_by_place = which;
    s->scales = a.scales;
    s->out = ga->out[which];
    s->part = ga->part[which];
    s->rank_major = which;
    s->runs = w.runs[which];
  };
  StreamArgs s = {};
  s.act = static_cast<const bf16*>(a.x);
  s.stride = a.x_stride;
  s.dim = a.in_dim;
  s.factor = vectors ? static_cast<const bf16*>(a.down) : nullptr;
  s.by_channel = back;
  s.planes = planes;
  s.off = a.off;
  s.perm = a.perm;
  s.check_word = a.check_word;
  s.n = a.n;
  s.G = a.G;
  s.rank = a.rank;
  s.runs = runs_for(a.n, a.G, blocks_of(a.in_dim, stream_channels(a.rank)), GPU_SMS, STREAM_ROWS, STREAM_RUN);
  if (back && ga->out[0]) outer(0, &s);
  cudaError_t e = cudaSuccess;
  if (s.factor || s.vec) e = launch_lowrank_stream(s, st);
  if (e != cudaSuccess || !vectors) return e;
  SumArgs u = {planes, blocks_of(a.in_dim, stream_channels(a.rank)), vec, a.v, a.off, a.perm, a.check_word, a.n, a.G, a.rank, a.segments > a.G};
  e = launch_lowrank_sum(u, st);
  if (e != cudaSuccess) return e;
  if (a.y) {
    UpArgs p = {};
    p.vec = vec;
    p.scales = a.scales;
    p.factor = static_cast<const bf16*>(a.up);
    p.by_rank = back;
    p.base = static_cast<const bf16*>(a.base);
    p.out = static_cast<bf16*>(a.y);
    p.stride = a.y_stride;
    p.dim = a.out_dim;
    p.off = a.off;
    p.perm = a.perm;
    p.check_word = a.check_word;
    p.n = a.n;
    p.G = a.G;
    p.segments = a.segments;
    p.rank = a.rank;
    p.runs = runs_for(a.n, a.segments, blocks_of(a.out_dim, stream_channels(a.rank)), GPU_SMS, STREAM_ROWS, UP_RUN);
    p.skip_none = a.skip_none;
    e = launch_lowrank_up(p, st);
    if (e != cudaSuccess) return e;
  }
  if (!back || !ga->out[1]) return cudaSuccess;
  StreamArgs x = s;
  x.act = static_cast<const bf16*>(ga->act[1]);
  x.stride = ga->stride[1];
  x.dim = ga->dim[1];
  x.factor = nullptr;
  outer(1, &x);
  x.early = 1;  // behind the sum of the vectors or the kernel that takes them up
  return launch_lowrank_stream(x, st);
}

int check_lowrank(const emoe_lowrank_desc* D, int n, const int32_t* ids, const int32_t* off) {
  if (!D || n <= 0 || D->in_dim <= 0 || D->out_dim <= 0 || D->rank <= 0) return EMOE_ERR_INVALID_ARG;
  if (D->n_adapters < 1 || D->n_adapters > EMOE_MAX_EXPERTS) return EMOE_ERR_INVALID_ARG;
  if ((ids == nullptr) == (off == nullptr)) return EMOE_ERR_INVALID_ARG;
  if ((D->x_stride && D->x_stride < D->in_dim) || (D->y_stride && D->y_stride < D->out_dim)) return EMOE_ERR_INVALID_ARG;
  if (!dtype_ok(D->dtype) || D->rank > EMOE_MAX_RANK) return EMOE_ERR_UNSUPPORTED;
  if (D->in_dim % 8 != 0 || D->out_dim % 8 != 0 || D->in_dim > LR_MAX_DIM || D->out_dim > LR_MAX_DIM) return EMOE_ERR_UNSUPPORTED;
  if (n > 0x7fffffff / 16) return EMOE_ERR_UNSUPPORTED;
  const int64_t vec = 16 / static_cast<int64_t>(dtype_size(D->dtype));
  if (D->x_stride % vec != 0 || D->y_stride % vec != 0) return EMOE_ERR_ALIGNMENT;
  if (!ptr_aligned(ids, 4) || !ptr_aligned(off, 4)) return EMOE_ERR_ALIGNMENT;
  return EMOE_OK;
}

}  // namespace
}  // namespace emoe

using namespace emoe;

#define EMOE_CALL(ctx, call)                                    \
  do {                                                          \
    const cudaError_t e__ = (call);                             \
    if (e__ != cudaSuccess) return ctx_cuda_fail(ctx, e__);     \
  } while (0)

extern "C" {

size_t emoe_lowrank_workspace_bytes(const emoe_lowrank_desc* desc, int n) {
  int32_t given = 0;
  if (check_lowrank(desc, n, &given, nullptr) != EMOE_OK) return 0;
  const size_t forward = lowrank_layout(*desc, n, false).total, backward = lowrank_layout(*desc, n, true).total;
  return forward > backward ? forward : backward;
}

int emoe_lowrank_forward(emoe_ctx* ctx, const emoe_lowrank_desc* desc, const void* A, const void* B, const float* scales, const void* x, int n,
                         const int32_t* ids, const int32_t* off, const void* base, void* y, float* out_v, void* stream) {
  const int rc = check_lowrank(desc, n, ids, off);
  if (rc != EMOE_OK) return rc;
  if (!A || !B || !x || !y) return EMOE_ERR_INVALID_ARG;
  if (!ptr_aligned(A, 16) || !ptr_aligned(B, 16) || !ptr_aligned(x, 16) || !ptr_aligned(base, 16) || !ptr_aligned(y, 16) ||
      !ptr_aligned(scales, 4) || !ptr_aligned(out_v, 16))
    return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LowrankArgs a = {};
  a.x = x;
  a.base = base;
  a.down = A;
  a.up = B;
  a.scales = scales;
  a.y = y;
  a.v = out_v;
  a.check_word = ctx_check_word(ctx);
  a.n = n;
  a.G = a.segments = desc->n_adapters;
  a.rank = desc->rank;
  a.in_dim = desc->in_dim;
  a.out_dim = desc->out_dim;
  a.skip_none = base == y;
  a.x_stride = static_cast<size_t>(desc->x_stride ? desc->x_stride : desc->in_dim);
  a.y_stride = static_cast<size_t>(desc->y_stride ? desc->y_stride : desc->out_dim);
  a.off = off;
  size_t have = 0;
  char* ws = ctx_workspace(ctx, &have);
  const LowrankLayout w = lowrank_layout(*desc, n, false);
  const bool streams = takes_stream(*desc, n, false);
  if (ids && n <= LR_IDS_ROWS && !streams) {
    a.ids = ids;
    a.segments = desc->n_adapters + 1;
  } else if (off && streams) {
    if (w.total > have) return EMOE_ERR_WORKSPACE;
  } else if (ids) {
    if ((streams ? w.total : w.vec) > have) return EMOE_ERR_WORKSPACE;
    int32_t *off_ws = reinterpret_cast<int32_t*>(ws + w.off), *perm = reinterpret_cast<int32_t*>(ws + w.perm);
    EMOE_CALL(ctx, launch_sort_pairs(ids, n, desc->n_adapters + 1, true, nullptr, off_ws, perm, true, nullptr, a.check_word, st));
    a.off = off_ws;
    a.perm = perm;
    a.segments = desc->n_adapters + 1;
  }
  if (streams) EMOE_CALL(ctx, launch_many(a, false, nullptr, ws, w, st));
  else EMOE_CALL(ctx, desc->dtype == EMOE_DTYPE_BF16 ? (launch_lowrank<__nv_bfloat16, false>(a, st)) : (launch_lowrank<float, false>(a, st)));
  return EMOE_OK;
}

int emoe_lowrank_backward(emoe_ctx* ctx, const emoe_lowrank_desc* desc, const void* A, const void* B, const float* scales, const void* x,
                          const void* dy, int n, const int32_t* ids, const int32_t* off, const float* v, const void* dx_base, void* dx, float* dA,
                          float* dB, void* stream) {
  const int rc = check_lowrank(desc, n, ids, off);
  if (rc != EMOE_OK) return rc;
  if (!dy || (!dx && !dA && !dB)) return EMOE_ERR_INVALID_ARG;
  if (((dx || dA) && !B) || (dx && !A) || (dA && !x) || (dB && !v)) return EMOE_ERR_INVALID_ARG;
  if (!ptr_aligned(A, 16) || !ptr_aligned(B, 16) || !ptr_aligned(x, 16) || !ptr_aligned(dy, 16) || !ptr_aligned(dx_base, 16) || !ptr_aligned(dx, 16) ||
      !ptr_aligned(dA, 16) || !ptr_aligned(dB, 16) || !ptr_aligned(scales, 4) || !ptr_aligned(v, 16))
    return EMOE_ERR_ALIGNMENT;
  if (!ctx) return EMOE_ERR_INVALID_ARG;
  size_t have = 0;
  char* ws = ctx_workspace(ctx, &have);
  const LowrankLayout w = lowrank_layout(*desc, n, true);
  const bool streams = takes_stream(*desc, n, true);
  if (w.total > have) return EMOE_ERR_WORKSPACE;
  const CallScope scope(ctx);
  EMOE_CALL(ctx, scope.error());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t *off_ws = reinterpret_cast<int32_t*>(ws + w.off), *perm = reinterpret_cast<int32_t*>(ws + w.perm);
  float* dv = reinterpret_cast<float*>(ws + w.vec);
  LowrankArgs a = {};
  a.x = dy;
  a.base = dx_base;
  a.down = B;
  a.up = A;
  a.scales = scales;
  a.y = dx;
  a.v = dA && !streams ? dv : nullptr;
  a.check_word = ctx_check_word(ctx);
  a.n = n;
  a.G = a.segments = desc->n_adapters;
  a.rank = desc->rank;
  a.in_dim = desc->out_dim;
  a.out_dim = desc->in_dim;
  a.skip_none = dx_base == dx;
  a.x_stride = static_cast<size_t>(desc->y_stride ? desc->y_stride : desc->out_dim);
  a.y_stride = static_cast<size_t>(desc->x_stride ? desc->x_stride : desc->in_dim);
  a.off = off;
  if (ids) {
    a.segments = desc->n_adapters + 1;
    if (n <= LR_IDS_ROWS && !streams && (dx || dA)) {
      a.ids = ids;
      a.off_out = off_ws;
      a.perm_out = perm;
    } else {
      EMOE_CALL(ctx, launch_sort_pairs(ids, n, desc->n_adapters + 1, true, nullptr, off_ws, perm, true, nullptr, a.check_word, st));
      a.off = off_ws;
      a.perm = perm;
    }
  }
  GradArgs ga = {};
  ga.act[0] = dy;
  ga.act[1] = x;
  ga.vec[0] = v;
  ga.vec[1] = dv;
  ga.stride[0] = a.x_stride;
  ga.stride[1] = a.y_stride;
  ga.dim[0] = desc->out_dim;
  ga.dim[1] = desc->in_dim;
  ga.out[0] = dB;
  ga.out[1] = dA;
  ga.scales = scales;
  ga.off = ids ? off_ws : off;
  ga.perm = ids ? perm : nullptr;
  ga.check_word = a.check_word;
  ga.n = n;
  ga.G = desc->n_adapters;
  ga.rank = desc->rank;
  for (int i = 0; i < 2; ++i) {
    ga.part[i] = reinterpret_cast<float*>(ws + w.part[i]);
    ga.blocks[i] = ga.out[i] ? blocks_of(ga.dim[i], GR_CHANNELS) : 0;
    ga.runs[i] = w.runs[i];
  }
  if (streams) {
    EMOE_CALL(ctx, launch_many(a, true, &ga, ws, w, st));
  } else {
    const bool bf16 = desc->dtype == EMOE_DTYPE_BF16;
    if (dx || dA) EMOE_CALL(ctx, bf16 ? (launch_lowrank<__nv_bfloat16, true>(a, st)) : (launch_lowrank<float, true>(a, st)));
    if (dA || dB) EMOE_CALL(ctx, bf16 ? launch_grads<__nv_bfloat16>(ga, st) : launch_grads<float>(ga, st));
  }
  if (dA || dB) EMOE_CALL(ctx, launch_join(ga, streams, off && !dx && !dA, st));
  return EMOE_OK;
}

}  // extern "C"

// Pieces that the kernels of the low-rank adapters share (lowrank.cu: few rows, fp32, the calls; lowrank_stream.cu: many bf16 rows).
#pragma once
#include "rows.cuh"

namespace emoe {

constexpr int LR_THREADS = 256, LR_WARPS = LR_THREADS / 32;

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// d = a . b, nothing added
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// Two fp32 values as N pairs of bf16 parts, largest first.  All parts but the last are truncated: what is left is exact, so three
// parts are the value itself.  Of two parts (bf16 results) an infinity is the first alone; of three (fp32 results) its rest is NaN, as is its
// product with any zero part of the other side (the test would be a third of the split).
template <int N>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    if (N == 2 && i == N - 1) {
      const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
      part[i] = *reinterpret_cast<const uint32_t*>(&r);
    } else {
      part[i] = __byte_perm(ua, ub, 0x7632);
    }
    a = N == 2 && isinf(a) ? 0.f : a - __uint_as_float(ua & 0xffff0000u);
    b = N == 2 && isinf(b) ? 0.f : b - __uint_as_float(ub & 0xffff0000u);
  }
}

template <typename T>
struct Parts {  // bf16 parts of a factor or activation, and of the fp32 vector it is multiplied with
  static constexpr int IN = sizeof(T) == 4 ? 3 : 1;
  static constexpr int VEC = sizeof(T) == 4 ? 3 : 2;
};

// N sums of products of parts side by side: d[k] (+)= a[k or 0] . b[k or 0].  The products of one sum wait for each other, some 35 clocks each,
// so that those of the others stand between them.
template <bool FIRST, int PA, int PB, int N, int NA, int NB>
__device__ __forceinline__ void mma_parts_of(float (&d)[N][4], const uint32_t (&a)[NA][PA][4], const uint32_t (&b)[NB][PB][2]) {
  bool first = FIRST;
#pragma unroll
  for (int i = PA - 1; i >= 0; --i)  // smallest first
#pragma unroll
    for (int j = PB - 1; j >= 0; --j)
      if (i + j < 3) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const uint32_t(&x)[4] = a[NA == 1 ? 0 : k][i];
          const uint32_t(&y)[2] = b[NB == 1 ? 0 : k][j];
          if (first) mma_bf16_first(d[k], x, y[0], y[1]);
          else mma_bf16(d[k], x, y[0], y[1]);
        }
        first = false;
      }
}

__device__ __forceinline__ uint4 load16(const void* p) {
  uint32_t w[4];
  load_words(p, w);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 load16_keep(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// The rows of segment i, off[i] .. off[i + 1] - 1, as far as there are such rows: the offsets are the caller's, and whatever they hold, both ends are
// cut to the rows before they are subtracted.
struct RowSpan {
  int begin, rows;
};
__device__ __forceinline__ RowSpan span_of(const int32_t* __restrict__ off, int i, int n) {
  const int begin = min(max(off[i], 0), n), end = min(max(off[i + 1], 0), n);
  return {begin, max(end - begin, 0)};
}
// Offsets that descend or leave the rows set the check word: one CTA of a call looks at them, in the fused kernel, the sum of the vectors or (dB alone) the join,
// which have registers to spare.
__device__ __forceinline__ void check_offsets(const int32_t* __restrict__ off, int segments, int n, int* check_word) {
  bool bad = false;
#pragma unroll 1
  for (int i = threadIdx.x; i < segments; i += blockDim.x) bad |= off[i] < 0 || off[i + 1] < off[i] || off[i + 1] > n;
  if (bad) atomicOr(check_word, CHECK_BAD_EXPERT_ID);
}

// ---- rows shared out evenly ----------------------------------------------------------------------
// The rows of every segment (the G adapters and, where there is one more, the rows of none) make tiles of H rows, the last of a
// segment with fewer; the tiles of all segments, one behind the other, are cut into even runs, one per CTA.  A run may begin and end
// inside a segment.
constexpr int MAX_SEGMENTS = EMOE_MAX_EXPERTS + 1;
struct TileList {
  int first[MAX_SEGMENTS + 1];  // of a segment's tiles; behind the last: their number
  int begin[MAX_SEGMENTS];      // of its rows, in the order
  int rows[MAX_SEGMENTS];
  int scan[LR_WARPS];
  int segment;                  // of the CTA's first tile
};
struct TileRun {
  int lo, hi, per;  // tiles of this CTA; of every CTA but the last
};

// Fills the list and gives run `cta` of `ctas`.  Every thread of the CTA calls it (at least LR_THREADS).
template <int H>
__device__ __forceinline__ TileRun list_tiles(TileList& list, const int32_t* __restrict__ off, int segments, int n, int cta, int ctas) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const auto segment = [&](int i) {
    const RowSpan span = span_of(off, i, n);
    list.begin[i] = span.begin;
    list.rows[i] = span.rows;
    return (span.rows + H - 1) / H;
  };
  const int tiles = tid < min(segments, LR_THREADS) ? segment(tid) : 0;
  int last = 0;
  if (tid == 0 && segments > LR_THREADS) last = segment(LR_THREADS);  // a 257th segment: beside 256 adapters
  int incl = tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31 && warp < LR_WARPS) list.scan[warp] = incl;
  __syncthreads();
  int front = 0, all = 0;
#pragma unroll
  for (int w = 0; w < LR_WARPS; ++w) {
    if (w < warp) front += list.scan[w];
    all += list.scan[w];
  }
  if (tid < min(segments, LR_THREADS)) list.first[tid] = front + incl - tiles;
  if (tid == 0) {
    list.first[min(segments, LR_THREADS)] = all;
    if (segments > LR_THREADS) list.first[segments] = all + last;
  }
  __syncthreads();
  const int total = list.first[segments], per = max((total + ctas - 1) / ctas, 1), lo = min(cta * per, total);
  for (int i = tid; i < segments; i += blockDim.x)
    if (lo >= list.first[i] && lo < list.first[i + 1]) list.segment = i;
  __syncthreads();
  return {lo, min(lo + per, total), per};
}
struct Tile {
  int begin, rows;    // in the order
  bool starts, ends;  // the first, the last of its segment within the run
};
// A walk along a run, tile by tile; `segment` is that of the last tile given.
template <int H>
struct RunWalk {
  const TileList& list;
  int lo, hi, at, segment;
  __device__ __forceinline__ RunWalk(const TileList& l, const TileRun& run) : list(l), lo(run.lo), hi(run.hi), at(run.lo), segment(l.segment) {}
  __device__ __forceinline__ bool more() const { return at < hi; }
  __device__ __forceinline__ int next_segment() const {  // while there is more
    int s = segment;
    while (at >= list.first[s + 1]) ++s;
    return s;
  }
  __device__ __forceinline__ Tile next() {
    segment = next_segment();
    const int first = list.first[segment], in_segment = (at - first) * H;
    const Tile t = {list.begin[segment] + in_segment, min(H, list.rows[segment] - in_segment), at == lo || at == first,
                    at + 1 == hi || at + 1 == list.first[segment + 1]};
    ++at;
    return t;
  }
};
// Lists the rows of a run of tiles of H rows: place (t - lo) * H + i holds row i of tile t, -1 beyond its last and (none_too false) for rows of no adapter.
template <int H>
__device__ __forceinline__ void list_rows(const TileList& list, const TileRun& run, const int32_t* __restrict__ perm, int G, bool none_too, int* s_rows) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int t = run.lo + warp, s = list.segment; t < run.hi; t += warps) {
    while (t >= list.first[s + 1]) ++s;
    const int in_segment = (t - list.first[s]) * H, begin = list.begin[s] + in_segment, rows = s >= G && !none_too ? 0 : list.rows[s] - in_segment;
    for (int i = lane; i < H; i += 32) s_rows[(t - run.lo) * H + i] = i >= rows ? -1 : perm ? perm[begin + i] : begin + i;
  }
}
// Outer products of a segment that several runs share are joined behind the kernel, in order.  Where a run leaves its share of segment
// s: the part of one that goes on in the next run, else of one that began before; -1: the segment is the run's alone.
__device__ __forceinline__ int share_of(const TileList& list, const TileRun& run, int s, int cta) {
  if (list.first[s + 1] > run.hi) return 2 * cta + 1;
  return list.first[s] < run.lo ? 2 * cta : -1;
}

// ---- many bf16 rows (lowrank_stream.cu) --------------------------------------------------------

// channels of a CTA: as many as tensor memory has room for
__host__ __device__ constexpr int stream_channels(int rank) { return rank <= 32 ? 512 : 256; }
// Rows of their tiles, the unit of a run (finer runs, even in rows, cut more tiles short, and a short one costs little less than a full one: 16
// rows 83 us where 128 rows take 75, 4099 rows of 16 adapters); tiles of the longest run, which is how many products are added in tensor memory, and how
// many rows a CTA lists.
constexpr int STREAM_ROWS = 128, STREAM_RUN = 8, UP_RUN = 16;

struct StreamArgs {
  const __nv_bfloat16* act;     // rows that go by
  size_t stride;
  int dim;                      // values per row, a multiple of 8
  const __nv_bfloat16* factor;  // down factor, [rank][dim] or (by_channel) [dim][rank]; null: no low-rank vectors
  int by_channel;
  float* planes;                // [blocks of stream_channels][n][rank], by place in the order: shares of the low-rank vectors
  const float* vec;             // vectors of the outer products, [..][rank]; null: none
  int vec_by_place;             // by place in the order, else by row
  const float* scales;          // of the vectors; null: 1
  float *out, *part;            // [adapters][dim][rank] or (rank_major) [rank][dim]; shares of segments that several runs have
  int rank_major;
  const int32_t *off, *perm;    // perm null: places are rows
  int* check_word;
  int n, G, rank, runs;
  int early;                    // all inputs but the vectors are older than the kernel in front, which waited before its trigger
};
cudaError_t launch_lowrank_stream(const StreamArgs& a, cudaStream_t st);

struct SumArgs {
  const float* planes;
  int count;         // planes
  float* by_place;   // [n][rank]
  float* by_row;     // null: not wanted
  const int32_t *off, *perm;
  int* check_word;
  int n, G, rank, with_none;  // with_none: the rows behind the last adapter's get zeros
};
cudaError_t launch_lowrank_sum(const SumArgs& a, cudaStream_t st);

struct UpArgs {
  const float* vec;             // [n][rank] by place
  const float* scales;
  const __nv_bfloat16* factor;  // up factor, [dim][rank] or (by_rank) [rank][dim]
  int by_rank;
  const __nv_bfloat16* base;    // null: zeros
  __nv_bfloat16* out;
  size_t stride;
  int dim;
  const int32_t *off, *perm;
  int* check_word;
  int n, G, segments, rank, runs, skip_none;
};
// directly behind launch_lowrank_sum: all inputs but the vectors are older than that kernel
cudaError_t launch_lowrank_up(const UpArgs& a, cudaStream_t st);

}  // namespace emoe

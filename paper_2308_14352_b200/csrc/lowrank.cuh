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
// parts are the value itself.  An infinity has no rest.
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
    a = isinf(a) ? 0.f : a - __uint_as_float(ua & 0xffff0000u);
    b = isinf(b) ? 0.f : b - __uint_as_float(ub & 0xffff0000u);
  }
}

template <typename T>
struct Parts {  // bf16 parts of a factor or activation, and of the fp32 vector it is multiplied with
  static constexpr int IN = sizeof(T) == 4 ? 3 : 1;
  static constexpr int VEC = sizeof(T) == 4 ? 3 : 2;
};

// a . b over the kept products of their parts
template <int PA, int PB>
__device__ __forceinline__ void mma_parts(float (&d)[4], const uint32_t (&a)[PA][4], const uint32_t (&b)[PB][2]) {
#pragma unroll
  for (int i = PA - 1; i >= 0; --i)  // smallest first
#pragma unroll
    for (int j = PB - 1; j >= 0; --j)
      if (i + j < 3) mma_bf16(d, a[i], b[j][0], b[j][1]);
}

__device__ __forceinline__ uint4 load16(const void* p) {
  uint32_t w[4];
  load_words(p, w);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 load16_keep(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// A run of one adapter's rows: adapter (-1: the rows of no adapter), first place in the order and rows, the number of its
// adapter's chunks and its place among the chunks of adapters with several.
struct Chunk {
  int adapter, begin, rows, of_adapter, place;
};
constexpr int CHUNK_SCAN = 2 * LR_WARPS + 5;

// Chunk `c` of the list of all segments' chunks of `chunk_rows` rows; false: no such chunk.  Segments: the G adapters and, where there is
// one more, the rows of none.  Every thread of the CTA calls it; s_scan: CHUNK_SCAN words.
__device__ __forceinline__ bool find_chunk(const int32_t* __restrict__ off, int segments, int G, int n, int chunk_rows, int c, int* s_scan, Chunk* out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const auto segment = [&](int i, int* begin) {
    *begin = min(max(off[i], 0), n);
    return max(min(off[i + 1], n) - *begin, 0);
  };
  int begin = 0, rows = 0, last_begin = 0, last_rows = 0;
  if (tid < min(segments, LR_THREADS)) rows = segment(tid, &begin);
  if (segments > LR_THREADS) last_rows = segment(LR_THREADS, &last_begin);  // a 257th segment: beside 256 adapters
  const int chunks = (rows + chunk_rows - 1) / chunk_rows, several = chunks > 1 && tid < G ? chunks : 0;
  int i0 = chunks, i1 = several;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u0 = __shfl_up_sync(0xffffffffu, i0, o), u1 = __shfl_up_sync(0xffffffffu, i1, o);
    if (lane >= o) {
      i0 += u0;
      i1 += u1;
    }
  }
  if (lane == 31 && warp < LR_WARPS) {  // (more threads than that have no segment)
    s_scan[warp] = i0;
    s_scan[LR_WARPS + warp] = i1;
  }
  int* s = s_scan + 2 * LR_WARPS;
  if (tid == 0) s[2] = 0;
  __syncthreads();
  int f0 = i0 - chunks, f1 = i1 - several, all = 0;
  for (int w = 0; w < LR_WARPS; ++w) {
    if (w < warp) {
      f0 += s_scan[w];
      f1 += s_scan[LR_WARPS + w];
    }
    all += s_scan[w];
  }
  const auto put = [&](int adapter, int first, int of, int begin_, int rows_, int place) {
    s[0] = adapter;
    s[1] = begin_ + (c - first) * chunk_rows;
    s[2] = min(chunk_rows, rows_ - (c - first) * chunk_rows);
    s[3] = of;
    s[4] = place;
  };
  if (c >= f0 && c < f0 + chunks) put(tid < G ? tid : -1, f0, chunks, begin, rows, f1 + (c - f0));
  const int last_chunks = (last_rows + chunk_rows - 1) / chunk_rows;
  if (tid == 0 && c >= all && c < all + last_chunks) put(-1, all, last_chunks, last_begin, last_rows, 0);
  __syncthreads();
  *out = {s[0], s[1], s[2], s[3], s[4]};
  return s[2] > 0;
}

// ---- many bf16 rows (lowrank_stream.cu) --------------------------------------------------------

constexpr int UP_CHANNELS = 64 * LR_WARPS;  // channels of a CTA of the up kernel
// ... of the stream kernel: as many as tensor memory has room for, beside the low-rank vectors
__host__ __device__ constexpr int stream_channels(int rank) { return rank <= 32 ? 512 : 256; }
constexpr int STREAM_ROWS = 128;             // rows of its tiles
constexpr int STREAM_MOST = 1024;            // most rows of a chunk: also how many products it adds in tensor memory before they are rounded properly

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
  float *out, *part;            // [adapters][dim][rank] or (rank_major) [rank][dim]; chunks of adapters with several
  int rank_major;
  const int32_t *off, *perm;    // perm null: places are rows
  int* check_word;
  int n, G, rank, chunk_rows, places;
};
cudaError_t launch_lowrank_stream(const StreamArgs& a, int chunks, cudaStream_t st);

struct SumArgs {
  const float* planes;
  int count;         // planes
  float* by_place;   // [n][rank]
  float* by_row;     // null: not wanted
  const int32_t *off, *perm;
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
  int n, G, segments, rank, chunk_rows, skip_none;
};
cudaError_t launch_lowrank_up(const UpArgs& a, int chunks, cudaStream_t st);

}  // namespace emoe

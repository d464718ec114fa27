// Low-rank adapters on many bf16 rows.  Three kernels that each read their activations once:
//   stream  x (dy) goes by: shares of the low-rank vectors v = A x (B^T dy), and in the backward pass, from the same
//           tiles, the outer products with the vectors of the other side, dB = s sum dy v^T (dA = sum dv x^T)
//   sum     the shares of the vectors, one per 512 channels, added in order
//   up      y = base + s B v (dx = dx_base + A^T s dv)
// A CTA owns 512 channels of a chunk of one adapter's rows, a warp 64 of them.  Its part of the factor, or of the outer
// products, stays in registers for all rows of the chunk, and the rows come as tiles of 16 x 64 values through a ring of its own in
// shared memory that cp.async fills some stages ahead: no wait among the warps for data, and memory latency costs no registers.
// The tiles are swizzled so that ldmatrix reads them both ways (rows for v, columns for the outer products) without bank conflicts.
#include "lowrank.cuh"

namespace emoe {
namespace {

constexpr int TILE_BYTES = 16 * 128;  // 16 rows of 64 bf16 values

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool live) {
  const int bytes = live ? 16 : 0;  // none: the place is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// byte of piece `p` (16 bytes) of row `r` in a tile
__device__ __forceinline__ uint32_t tile_at(int r, int p) { return r * 128 + ((p ^ (r & 7)) << 4); }

// One warp's ring of tiles.  Rows of the chunk beyond its end, and channels beyond the row's, read as zeros.
template <int STAGES>
struct Ring {
  uint32_t base;
  const __nv_bfloat16* src;
  size_t stride;
  const int* s_rows;
  int rows, lane;
  bool piece_live;

  __device__ __forceinline__ void init(const void* smem, const __nv_bfloat16* act, size_t stride_, int c0, int dim, const int* rows_list, int n_rows) {
    lane = threadIdx.x & 31;
    base = smem_addr(smem);
    piece_live = c0 + (lane & 7) * 8 < dim;
    src = act + (piece_live ? c0 + (lane & 7) * 8 : 0);
    stride = stride_;
    s_rows = rows_list;
    rows = n_rows;
  }
  // asks for stage `i` (16 rows); beyond the last row an empty group, so that the counts of waits hold
  __device__ __forceinline__ void ask(int i) {
    if (i * 16 < rows) {
      const uint32_t dst = base + i % STAGES * TILE_BYTES;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = (lane >> 3) + 4 * j, at = i * 16 + r;
        const bool live = piece_live && at < rows;
        copy_async16(dst + tile_at(r, lane & 7), src + static_cast<size_t>(live ? s_rows[at] : s_rows[0]) * stride, live);
      }
    }
    copy_commit();
  }
  // stage `i` is there for the whole warp, and the place of the one before is free
  __device__ __forceinline__ uint32_t get(int i) {
    copy_wait<STAGES - 2>();
    __syncwarp();
    return base + i % STAGES * TILE_BYTES;
  }
};

// Low-rank vectors of `ROWS` rows as bf16 parts, [PARTS][ROWS] rows of V_BYTES: eight neighbouring rows meet no bank twice.
template <int RT, int PARTS, int ROWS>
struct Vectors {
  static constexpr int RP = RT * 16, V_BYTES = RP * 2 + 16, BYTES = PARTS * ROWS * V_BYTES;
  static constexpr int PER_THREAD = ROWS * RP / 2 / LR_THREADS > 0 ? ROWS * RP / 2 / LR_THREADS : 1;  // pairs of neighbouring ranks
  float2 held[PER_THREAD];

  // rows [first, first + ROWS) of the chunk; row_of(i): the vector's row
  template <typename F>
  __device__ __forceinline__ void ask(const float* vec, int rank, int first, int rows, F&& row_of) {
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
      const int i = j * LR_THREADS + threadIdx.x, row = i / (RP / 2), r = i % (RP / 2) * 2;
      held[j] = make_float2(0.f, 0.f);
      if (row < ROWS && first + row < rows) {
        const float* v = vec + static_cast<size_t>(row_of(first + row)) * rank;
        if (r < rank) held[j].x = v[r];
        if (r + 1 < rank) held[j].y = v[r + 1];
      }
    }
  }
  __device__ __forceinline__ void put(char* buf, float scale) {
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
      const int i = j * LR_THREADS + threadIdx.x, row = i / (RP / 2), r = i % (RP / 2) * 2;
      if (row >= ROWS) continue;
      uint32_t p[PARTS];
      split_pair<PARTS>(scale * held[j].x, scale * held[j].y, p);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) *reinterpret_cast<uint32_t*>(buf + (k * ROWS + row) * V_BYTES + r * 2) = p[k];
    }
  }
};

template <int RT>
struct Stream {
  static constexpr int RP = RT * 16, ROWS = RT == 4 ? 16 : 32;  // rows between two meetings of the warps
  static constexpr int STAGES = 4;
  using Vec = Vectors<RT, 3, ROWS>;
  static constexpr int SUM_FLOATS = LR_WARPS * ROWS * RP;
  static constexpr size_t smem(bool down, bool outer, int chunk_rows) {
    return static_cast<size_t>(LR_WARPS) * STAGES * TILE_BYTES + (down ? sizeof(float) * SUM_FLOATS : 0) + (outer ? 2 * Vec::BYTES : 0) +
           sizeof(int) * chunk_rows;
  }
};
constexpr int ST_MAX_CHUNK = 2048;  // rows listed in shared memory

template <int RT, bool DOWN, bool OUTER>
__global__ void __launch_bounds__(LR_THREADS, RT == 1 ? 2 : 1) lowrank_stream_kernel(StreamArgs a) {
  using S = Stream<RT>;
  using Vec = typename S::Vec;
  constexpr int RP = S::RP, ROWS = S::ROWS, NR = 2 * RT;
  extern __shared__ __align__(128) char smem[];
  char* s_ring = smem;
  float* s_sum = reinterpret_cast<float*>(smem + LR_WARPS * S::STAGES * TILE_BYTES);  // [warp][row][rank]
  char* s_vec = reinterpret_cast<char*>(s_sum + (DOWN ? S::SUM_FLOATS : 0));
  int* s_rows = reinterpret_cast<int*>(s_vec + (OUTER ? 2 * Vec::BYTES : 0));
  __shared__ int s_scan[CHUNK_SCAN];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  pdl_wait();
  pdl_trigger();
  Chunk ch;
  if (!find_chunk(a.off, a.G, a.G, a.n, a.chunk_rows, blockIdx.x, s_scan, &ch)) return;
  if (OUTER && ch.of_adapter > 1 && ch.place >= a.places) {  // only where the segments overlap
    if (tid == 0) atomicOr(a.check_word, CHECK_BAD_EXPERT_ID);
    return;
  }
  for (int i = tid; i < ch.rows; i += LR_THREADS) s_rows[i] = a.perm ? a.perm[ch.begin + i] : ch.begin + i;
  __syncthreads();
  const int c0 = blockIdx.y * ST_CHANNELS + warp * 64;
  Ring<S::STAGES> ring;
  ring.init(s_ring + warp * S::STAGES * TILE_BYTES, a.act, a.stride, c0, a.dim, s_rows, ch.rows);
  for (int i = 0; i < S::STAGES - 1; ++i) ring.ask(i);

  // this warp's part of the down factor: [4 x 16 channels][rank in eights], columns are ranks.  by_channel: a word of B holds two
  // ranks of one channel, so column c of the tiles 2 s and 2 s + 1 is rank 16 s + 2 c and the one behind it.
  uint32_t down[DOWN ? 4 : 1][NR][2];
  if constexpr (DOWN) {
    const uint16_t* f = reinterpret_cast<const uint16_t*>(a.factor) + static_cast<size_t>(ch.adapter) * a.rank * a.dim;
    const bool even = a.rank % 2 == 0;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int c = c0 + kk * 16 + half * 8 + 2 * q;  // two channels
        if (a.by_channel) {
#pragma unroll
          for (int s = 0; s < RT; ++s) {
            const int r = 16 * s + 2 * g;
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (c < a.dim) {
                const uint16_t* p = f + static_cast<size_t>(c + j) * a.rank + r;
                if (even) {
                  if (r < a.rank) w[j] = *reinterpret_cast<const uint32_t*>(p);
                } else {
                  if (r < a.rank) w[j] = p[0];
                  if (r + 1 < a.rank) w[j] |= static_cast<uint32_t>(p[1]) << 16;
                }
              }
            down[kk][2 * s][half] = __byte_perm(w[0], w[1], 0x5410);
            down[kk][2 * s + 1][half] = __byte_perm(w[0], w[1], 0x7632);
          }
        } else {
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            const int r = nr * 8 + g;
            down[kk][nr][half] = r < a.rank && c < a.dim ? *reinterpret_cast<const uint32_t*>(f + static_cast<size_t>(r) * a.dim + c) : 0u;
          }
        }
      }
  }
  const float scale = OUTER && a.scales ? a.scales[ch.adapter] : 1.f;
  const auto row_of = [&](int i) { return a.vec_by_place ? ch.begin + i : s_rows[i]; };
  Vec vec;
  if constexpr (OUTER) {
    vec.ask(a.vec, a.rank, 0, ch.rows, row_of);
    vec.put(s_vec, scale);
  }
  float acc[OUTER ? 4 : 1][OUTER ? NR : 1][4] = {};
  int buf = 0;
  for (int r0 = 0; r0 < ch.rows; r0 += ROWS, buf ^= 1) {
    __syncthreads();  // the vectors of these rows are there, the sums of those before have been taken
    if constexpr (OUTER) vec.ask(a.vec, a.rank, r0 + ROWS, ch.rows, row_of);
    const uint32_t vecs = smem_addr(s_vec + buf * Vec::BYTES);
#pragma unroll
    for (int k = 0; k < ROWS / 16; ++k) {
      const int stage = r0 / 16 + k;
      if (stage * 16 >= ch.rows) break;
      const uint32_t tile = ring.get(stage);
      ring.ask(stage + S::STAGES - 1);
      if constexpr (DOWN) {
        float d[NR][4] = {};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t af[4];
          ldmatrix4(af, tile + tile_at((lane & 7) + (lane >> 3 & 1) * 8, 2 * kk + (lane >> 4)));
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) mma_bf16(d[nr], af, down[kk][nr][0], down[kk][nr][1]);
        }
        float* sum = s_sum + (warp * ROWS + k * 16 + g) * RP;
#pragma unroll
        for (int s = 0; s < RT; ++s) {
          if (a.by_channel) {  // columns 2 q and 2 q + 1 of both tiles: four neighbouring ranks
            *reinterpret_cast<float4*>(sum + 16 * s + 4 * q) = make_float4(d[2 * s][0], d[2 * s + 1][0], d[2 * s][1], d[2 * s + 1][1]);
            *reinterpret_cast<float4*>(sum + 8 * RP + 16 * s + 4 * q) = make_float4(d[2 * s][2], d[2 * s + 1][2], d[2 * s][3], d[2 * s + 1][3]);
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              *reinterpret_cast<float2*>(sum + 16 * s + 8 * h + 2 * q) = make_float2(d[2 * s + h][0], d[2 * s + h][1]);
              *reinterpret_cast<float2*>(sum + 8 * RP + 16 * s + 8 * h + 2 * q) = make_float2(d[2 * s + h][2], d[2 * s + h][3]);
            }
          }
        }
      }
      if constexpr (OUTER) {
        uint32_t vf[3][RT][4];  // two tiles of eight ranks each: b0, b1, b0, b1
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
          for (int s = 0; s < RT; ++s)
            ldmatrix4_t(vf[p][s], vecs + (p * ROWS + k * 16 + (lane & 7) + (lane >> 3 & 1) * 8) * Vec::V_BYTES + (2 * s + (lane >> 4)) * 16);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          uint32_t af[4];
          ldmatrix4_t(af, tile + tile_at((lane & 7) + (lane >> 4) * 8, 2 * m + (lane >> 3 & 1)));
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            // the tensor cores cut what they add: sixteen rows are summed by themselves, then added with rounding
            float d[4] = {};
#pragma unroll
            for (int p = 2; p >= 0; --p) mma_bf16(d, af, vf[p][nr / 2][nr % 2 * 2], vf[p][nr / 2][nr % 2 * 2 + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][nr][i] += d[i];
          }
        }
      }
    }
    if constexpr (OUTER) vec.put(s_vec + (buf ^ 1) * Vec::BYTES, scale);
    if constexpr (DOWN) {
      __syncthreads();
      // this CTA's share of the rows' vectors
      float* plane = a.planes + (static_cast<size_t>(blockIdx.y) * a.n + ch.begin + r0) * a.rank;
      const int rows = min(ROWS, ch.rows - r0);
      for (int i = tid; i < rows * RP; i += LR_THREADS) {
        const int row = i / RP, r = i % RP;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < LR_WARPS; ++w) v += s_sum[w * ROWS * RP + i];
        if (r < a.rank) plane[row * a.rank + r] = v;
      }
    }
  }
  if constexpr (OUTER) {
    const size_t size = static_cast<size_t>(a.dim) * a.rank;
    float* out = ch.of_adapter == 1 ? a.out + ch.adapter * size : a.part + ch.place * size;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = c0 + m * 16 + h * 8 + g;
        if (c >= a.dim) continue;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int r = nr * 8 + 2 * q + b;
            if (r < a.rank) out[a.rank_major ? static_cast<size_t>(r) * a.dim + c : static_cast<size_t>(c) * a.rank + r] = acc[m][nr][2 * h + b];
          }
      }
  }
}

__global__ void __launch_bounds__(256) lowrank_sum_kernel(SumArgs a) {
  pdl_wait();
  pdl_trigger();
  const size_t total = static_cast<size_t>(a.n) * a.rank;
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= total) return;
  const int place = static_cast<int>(i / a.rank), r = static_cast<int>(i % a.rank);
  const bool mine = place >= a.off[0] && place < a.off[a.G];
  if (!mine && !a.with_none) return;
  float v = 0.f;
  if (mine) {
#pragma unroll 8
    for (int p = 0; p < a.count; ++p) v += a.planes[p * total + i];
  }
  a.by_place[i] = v;
  if (a.by_row) a.by_row[static_cast<size_t>(a.perm ? a.perm[place] : place) * a.rank + r] = v;
}

template <int RT>
struct Up {
  static constexpr int ROWS = 64, STAGES = 5;
  using Vec = Vectors<RT, 2, ROWS>;
  static constexpr size_t smem(int chunk_rows) {
    return static_cast<size_t>(LR_WARPS) * STAGES * TILE_BYTES + 2 * Vec::BYTES + sizeof(int) * chunk_rows;
  }
};

// y = base + s B v.  Of the result's columns a lane owns eight neighbouring channels of two rows, so that base is read from the tile and y
// written in words of 16 bytes: column c of the tile i of four stands for the channel 8 (c / 2) + 2 i + c % 2 of 32.
template <int RT>
__global__ void __launch_bounds__(LR_THREADS, RT == 4 ? 1 : 2) lowrank_up_kernel(UpArgs a) {
  using U = Up<RT>;
  using Vec = typename U::Vec;
  extern __shared__ __align__(128) char smem[];
  char* s_vec = smem + LR_WARPS * U::STAGES * TILE_BYTES;
  int* s_rows = reinterpret_cast<int*>(s_vec + 2 * Vec::BYTES);
  __shared__ int s_scan[CHUNK_SCAN];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  pdl_wait();
  pdl_trigger();
  Chunk ch;
  if (!find_chunk(a.off, a.segments, a.G, a.n, a.chunk_rows, blockIdx.x, s_scan, &ch)) return;
  if (ch.adapter < 0 && a.skip_none) return;
  for (int i = tid; i < ch.rows; i += LR_THREADS) s_rows[i] = a.perm ? a.perm[ch.begin + i] : ch.begin + i;
  __syncthreads();
  const int c0 = blockIdx.y * ST_CHANNELS + warp * 64;
  Ring<U::STAGES> ring;
  ring.init(smem + warp * U::STAGES * TILE_BYTES, a.base, a.stride, c0, a.base ? a.dim : 0, s_rows, ch.rows);
  if (a.base)
    for (int i = 0; i < U::STAGES - 1; ++i) ring.ask(i);

  uint32_t up[RT][2][4][2];  // [16 ranks][32 channels][8 of them][k half]
#pragma unroll
  for (int s = 0; s < RT; ++s)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = 16 * s + 8 * half + 2 * q, c8 = c0 + 32 * h + 8 * (g >> 1);  // two ranks, eight channels
        if (ch.adapter < 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) up[s][h][i][half] = 0;
        } else if (a.by_rank) {
          const __nv_bfloat16* f = a.factor + static_cast<size_t>(ch.adapter) * a.rank * a.dim;
          uint4 w[2];
#pragma unroll
          for (int j = 0; j < 2; ++j)
            w[j] = r + j < a.rank && c8 < a.dim ? *reinterpret_cast<const uint4*>(f + static_cast<size_t>(r + j) * a.dim + c8) : make_uint4(0, 0, 0, 0);
          const uint32_t sel = (g & 1) ? 0x7632 : 0x5410;
          up[s][h][0][half] = __byte_perm(w[0].x, w[1].x, sel);
          up[s][h][1][half] = __byte_perm(w[0].y, w[1].y, sel);
          up[s][h][2][half] = __byte_perm(w[0].z, w[1].z, sel);
          up[s][h][3][half] = __byte_perm(w[0].w, w[1].w, sel);
        } else {
          const uint16_t* f = reinterpret_cast<const uint16_t*>(a.factor) + static_cast<size_t>(ch.adapter) * a.rank * a.dim;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = c8 + 2 * i + (g & 1);
            uint32_t w = 0;
            if (c < a.dim) {
              const uint16_t* p = f + static_cast<size_t>(c) * a.rank + r;
              if (a.rank % 2 == 0) {
                if (r < a.rank) w = *reinterpret_cast<const uint32_t*>(p);
              } else {
                if (r < a.rank) w = p[0];
                if (r + 1 < a.rank) w |= static_cast<uint32_t>(p[1]) << 16;
              }
            }
            up[s][h][i][half] = w;
          }
        }
      }
  const float scale = a.scales && ch.adapter >= 0 ? a.scales[ch.adapter] : 1.f;
  const auto row_of = [&](int i) { return ch.begin + i; };
  const int vec_rows = ch.adapter >= 0 ? ch.rows : 0;
  Vec vec;
  vec.ask(a.vec, a.rank, 0, vec_rows, row_of);
  vec.put(s_vec, scale);
  int buf = 0;
  for (int r0 = 0; r0 < ch.rows; r0 += U::ROWS, buf ^= 1) {
    __syncthreads();  // the vectors of these rows are there
    vec.ask(a.vec, a.rank, r0 + U::ROWS, vec_rows, row_of);
    const uint32_t vecs = smem_addr(s_vec + buf * Vec::BYTES);
#pragma unroll 1
    for (int k = 0; k < U::ROWS / 16; ++k) {
      const int stage = r0 / 16 + k;
      if (stage * 16 >= ch.rows) break;
      float d[2][4][4] = {};
#pragma unroll
      for (int s = 0; s < RT; ++s)
#pragma unroll
        for (int p = 1; p >= 0; --p) {
          uint32_t vf[4];
          ldmatrix4(vf, vecs + (p * U::ROWS + k * 16 + (lane & 7) + (lane >> 3 & 1) * 8) * Vec::V_BYTES + (2 * s + (lane >> 4)) * 16);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) mma_bf16(d[h][i], vf, up[s][h][i][0], up[s][h][i][1]);
        }
      uint32_t tile = 0;
      if (a.base) {
        tile = ring.get(stage);
        ring.ask(stage + U::STAGES - 1);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int row = g + 8 * half, at = stage * 16 + row;
        if (at >= ch.rows) continue;
        __nv_bfloat16* y = a.out + static_cast<size_t>(s_rows[at]) * a.stride;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = c0 + 32 * h + 8 * q;
          if (c >= a.dim) continue;
          Piece<__nv_bfloat16, 8> p = {};
          if (a.base)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[2]), "=r"(p.w[3])
                         : "r"(tile + tile_at(row, 4 * h + q))
                         : "memory");
          float f[8];
          widen<__nv_bfloat16, 8>(p, f);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f[2 * i] += d[h][i][2 * half];
            f[2 * i + 1] += d[h][i][2 * half + 1];
          }
          store_piece<__nv_bfloat16, 8>(y + c, narrow<__nv_bfloat16, 8>(f));
        }
      }
    }
    vec.put(s_vec + (buf ^ 1) * Vec::BYTES, scale);
  }
}

template <int RT, bool DOWN, bool OUTER>
cudaError_t launch_stream_of(const StreamArgs& a, int chunks, cudaStream_t st) {
  const cudaError_t e = allow_smem<lowrank_stream_kernel<RT, DOWN, OUTER>>(static_cast<int>(Stream<RT>::smem(DOWN, OUTER, ST_MAX_CHUNK)));
  if (e != cudaSuccess) return e;
  return launch_chain(lowrank_stream_kernel<RT, DOWN, OUTER>, dim3(chunks, (a.dim + ST_CHANNELS - 1) / ST_CHANNELS), dim3(LR_THREADS),
                      Stream<RT>::smem(DOWN, OUTER, a.chunk_rows), st, a);
}

template <int RT>
cudaError_t launch_stream_rank(const StreamArgs& a, int chunks, cudaStream_t st) {
  if (a.factor && a.vec) return launch_stream_of<RT, true, true>(a, chunks, st);
  return a.factor ? launch_stream_of<RT, true, false>(a, chunks, st) : launch_stream_of<RT, false, true>(a, chunks, st);
}

template <int RT>
cudaError_t launch_up_rank(const UpArgs& a, int chunks, cudaStream_t st) {
  const cudaError_t e = allow_smem<lowrank_up_kernel<RT>>(static_cast<int>(Up<RT>::smem(ST_MAX_CHUNK)));
  if (e != cudaSuccess) return e;
  return launch_chain(lowrank_up_kernel<RT>, dim3(chunks, (a.dim + ST_CHANNELS - 1) / ST_CHANNELS), dim3(LR_THREADS), Up<RT>::smem(a.chunk_rows), st, a);
}

}  // namespace

cudaError_t launch_lowrank_stream(const StreamArgs& a, int chunks, cudaStream_t st) {
  if (a.chunk_rows > ST_MAX_CHUNK) return cudaErrorInvalidValue;
  if (a.rank <= 16) return launch_stream_rank<1>(a, chunks, st);
  return a.rank <= 32 ? launch_stream_rank<2>(a, chunks, st) : launch_stream_rank<4>(a, chunks, st);
}

cudaError_t launch_lowrank_sum(const SumArgs& a, cudaStream_t st) {
  const size_t total = static_cast<size_t>(a.n) * a.rank;
  return launch_chain(lowrank_sum_kernel, dim3(static_cast<unsigned>((total + 255) / 256)), dim3(256), 0, st, a);
}

cudaError_t launch_lowrank_up(const UpArgs& a, int chunks, cudaStream_t st) {
  if (a.chunk_rows > ST_MAX_CHUNK) return cudaErrorInvalidValue;
  if (a.rank <= 16) return launch_up_rank<1>(a, chunks, st);
  return a.rank <= 32 ? launch_up_rank<2>(a, chunks, st) : launch_up_rank<4>(a, chunks, st);
}

}  // namespace emoe

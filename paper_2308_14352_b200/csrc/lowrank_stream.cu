// Low-rank adapters on many bf16 rows.  Three kernels that each read their activations once:
//   stream  x (dy) goes by: shares of the low-rank vectors v = A x (B^T dy), and in the backward pass, from the same
//           tiles, the outer products with the vectors of the other side, dB = s sum dy v^T (dA = sum dv x^T)
//   sum     the shares of the vectors, one per 512 channels, added in order
//   up      y = base + s B v (dx = dx_base + A^T s dv)
// stream: a value of x takes part in 16 to 64 multiply-adds of v and three times as many of the outer products, too much for the
// instructions that registers feed once the rank is 32 or 64, so its tiles go from cp.async (rows of any order) to tcgen05 and both sums
// stay in tensor memory; no thread touches a value of x.  A CTA owns 512 (256) channels of an even run of the rows.
// up: every value of base meets an fp32 sum in a register anyway, so the product is mma.sync there: a warp owns 64 channels, its part of
// the factor stays in registers, and base comes as tiles of 16 x 64 values through a ring of its own in shared memory that cp.async
// fills some stages ahead.
#include "lowrank.cuh"
#include "pipe.cuh"
#include "umma.cuh"

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

// One warp's ring of tiles.  Places without a row, and channels beyond the row's, read as zeros.
template <int STAGES>
struct Ring {
  uint32_t base;
  const __nv_bfloat16* src;
  size_t stride;
  const int* s_rows;
  int stages, lane;
  bool piece_live;

  __device__ __forceinline__ void init(const void* smem, const __nv_bfloat16* act, size_t stride_, int c0, int dim, const int* rows_list, int n_stages) {
    lane = threadIdx.x & 31;
    base = smem_addr(smem);
    piece_live = c0 + (lane & 7) * 8 < dim;
    src = act + (piece_live ? c0 + (lane & 7) * 8 : 0);
    stride = stride_;
    s_rows = rows_list;
    stages = n_stages;
  }
  // asks for stage `i` (16 rows); where there are none an empty group, so that the counts of waits hold
  __device__ __forceinline__ void ask(int i) {
    if (i < stages && s_rows[i * 16] >= 0) {
      const uint32_t dst = base + i % STAGES * TILE_BYTES;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = (lane >> 3) + 4 * j, row = s_rows[i * 16 + r];
        copy_async16(dst + tile_at(r, lane & 7), src + static_cast<size_t>(max(row, 0)) * stride, piece_live && row >= 0);
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

// ---- stream -------------------------------------------------------------------------------------

// Roles: warps 0-3 bring the factor and the vectors into shared memory as operands and carry results out of tensor memory, warps 4-7
// copy the rows, warp 8 issues the products.
constexpr int SK_THREADS = 288, SK_SIDE = 128, SK_STAGES = 4;
constexpr int SK_TILE = STREAM_ROWS * 128, SK_STAGE = 2 * SK_TILE;  // 128 rows x 64 values; a stage: 128 channels

template <int RT>
struct Stream {
  static constexpr int RP = RT * 16, CHANNELS = stream_channels(RP), PAIRS = CHANNELS / 128;
  static constexpr int FACTOR = CHANNELS / 64 * RP * 128;      // [rank][channels], K-major tiles of 64 channels
  static constexpr int VEC = 2 * 3 * RP * 128;                 // [three parts of rank][128 rows], K-major tiles of 64 rows
  static constexpr int VEC_BUFS = RT == 4 ? 1 : 2;
  static constexpr int COL_OUTER = 2 * RP, COLS = COL_OUTER + PAIRS * 3 * RP, TMEM = COLS <= 256 ? 256 : 512;
  static_assert(COLS <= 512, "tensor memory has 512 columns");
  static constexpr size_t smem(bool down, bool outer) {
    return 1024 + static_cast<size_t>(SK_STAGES) * SK_STAGE + (down ? FACTOR : 0) + (outer ? VEC_BUFS * VEC : 0) + sizeof(int) * STREAM_RUN * STREAM_ROWS + sizeof(TileList);
  }
};

// byte of value `k` of row `n` in K-major tiles of 64 values, `rows` rows each
__device__ __forceinline__ uint32_t kmajor_at(int n, int k, int rows) {
  return k / 64 * rows * 128 + n * 128 + ((k % 64 / 8 ^ (n & 7)) << 4) + k % 8 * 2;
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The products, for a tile X of 128 rows x 128 channels (two swizzled tiles of 64, as cp.async leaves them):
//   vectors [128 rows][rank]              += X F^T          X read along its rows (K-major), 16 channels per instruction
//   outer   [128 channels][3 x rank]      += X^T V          X read along its columns (MN-major), 16 rows per instruction
// V are the rows' vectors in three bf16 parts side by side, so that the three products cost one instruction; they are added at the
// end.  Both sums stay in tensor memory: the vectors over the CTA's channels, the outer products over the rows of a segment in its run.  The
// tensor cores cut what they add: a run is no longer than 1024 rows, which costs some 1e-6.
template <int RT, bool DOWN, bool OUTER>
__global__ void __launch_bounds__(SK_THREADS, 1) lowrank_stream_kernel(StreamArgs a) {
  using S = Stream<RT>;
  constexpr int RP = S::RP, PAIRS = S::PAIRS;
  extern __shared__ char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * SK_STAGES + 12];
  __shared__ uint32_t tmem_slot;
  __shared__ int wait_words[PIPE_WORDS];
  volatile int* abort_flag = wait_words + PIPE_ABORT;
  char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  char* s_factor = smem + SK_STAGES * SK_STAGE;
  char* s_vec = s_factor + (DOWN ? S::FACTOR : 0);
  int* s_rows = reinterpret_cast<int*>(s_vec + (OUTER ? S::VEC_BUFS * S::VEC : 0));
  TileList& list = *reinterpret_cast<TileList*>(s_rows + STREAM_RUN * STREAM_ROWS);
  const uint32_t full = smem_u32(bars), empty = full + 8 * SK_STAGES, d1_full = empty + 8 * SK_STAGES, d1_empty = d1_full + 16,
                 vec_full = d1_empty + 16, vec_empty = vec_full + 16, ready = vec_empty + 16, d2_full = ready + 8, d2_empty = d2_full + 8;
  const int tid = threadIdx.x, warp = uniform_warp();
  if (tid == 0) {
    for (int i = 0; i < SK_STAGES; ++i) {
      mbar_init(full + 8 * i, SK_SIDE);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(d1_full + 8 * i, 1);
      mbar_init(d1_empty + 8 * i, SK_SIDE);
      mbar_init(vec_full + 8 * i, SK_SIDE);
      mbar_init(vec_empty + 8 * i, 1);
    }
    mbar_init(ready, SK_SIDE);
    mbar_init(d2_full, 1);
    mbar_init(d2_empty, SK_SIDE);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    wait_words[PIPE_ABORT] = 0;
    wait_words[PIPE_FRONT] = a.early;
  }
  if (!a.early) pdl_wait();
  const TileRun run = list_tiles<STREAM_ROWS>(list, a.off, a.G, a.n, blockIdx.x, a.runs);
  if (run.lo >= run.hi) {
    pdl_wait();
    pdl_trigger();
    return;
  }
  if (run.hi - run.lo > STREAM_RUN) {  // only where the segments overlap
    pdl_wait();
    if (tid == 0) atomicOr(a.check_word, CHECK_BAD_EXPERT_ID);
    return;
  }
  for (int t = run.lo + warp, s = list.segment; t < run.hi; t += SK_THREADS / 32) {
    const Tile tile = tile_of<STREAM_ROWS>(list, run, t, &s);
    for (int i = tid & 31; i < STREAM_ROWS; i += 32)
      s_rows[(t - run.lo) * STREAM_ROWS + i] = i < tile.rows ? (a.perm ? a.perm[tile.begin + i] : tile.begin + i) : -1;
  }
  if (warp == 8) tmem_alloc(smem_u32(&tmem_slot), S::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int c0 = blockIdx.y * S::CHANNELS, tiles = run.hi - run.lo;
  const int pairs = min(PAIRS, (a.dim - c0 + 127) / 128);  // of 128 channels; what the last has too many reads as zeros
  int segment = list.segment;

  if (warp >= 4 && warp < 8) {
    // ---- rows: a thread copies 16 bytes of every eighth row of a tile; places without a row and channels beyond the end become zeros
    const int i = tid - 128, piece = i & 15, row0 = i >> 4;
    const uint32_t dst = smem_u32(smem) + (piece >> 3) * SK_TILE + row0 * 128 + (((piece & 7) ^ row0) << 4);
    const __nv_bfloat16* row[STREAM_ROWS / 8];
    int it = 0;
    bool ok = true;
    const auto landed = [&](int stage) {
      fence_async_proxy();
      mbar_arrive(full + 8 * (stage % SK_STAGES));
    };
    for (int t = 0; t < tiles && ok; ++t) {
      uint32_t live = 0;
#pragma unroll
      for (int j = 0; j < STREAM_ROWS / 8; ++j) {
        const int r = s_rows[t * STREAM_ROWS + row0 + 8 * j];
        if (r >= 0) live |= 1u << j;
        row[j] = a.act + static_cast<size_t>(max(r, 0)) * a.stride;
      }
      for (int p = 0; p < pairs; ++p, ++it) {
        const int s = it % SK_STAGES, c = c0 + p * 128 + piece * 8;
        ok = mbar_wait(empty + 8 * s, ((it / SK_STAGES) & 1) ^ 1, a.check_word, abort_flag);
        if (!ok) break;
        const bool inside = c < a.dim;
#pragma unroll
        for (int j = 0; j < STREAM_ROWS / 8; ++j) copy_async16(dst + s * SK_STAGE + j * 1024, row[j] + (inside ? c : 0), inside && (live >> j & 1u));
        copy_commit();
        copy_wait<SK_STAGES - 1>();
        if (it >= SK_STAGES - 1) landed(it - (SK_STAGES - 1));
      }
    }
    copy_wait<0>();
    if (ok)
      for (int s = max(0, it - (SK_STAGES - 1)); s < it; ++s) landed(s);
  } else if (warp == 8) {
    // ---- products
    const uint32_t on = elect_one();
    constexpr uint32_t BF16_F32 = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);  // bf16 x bf16 -> fp32, M = 128
    constexpr uint32_t ID_DOWN = BF16_F32 | (static_cast<uint32_t>(RP / 8) << 17), ID_OUTER = BF16_F32 | (1u << 15) | (static_cast<uint32_t>(3 * RP / 8) << 17);
    const uint32_t ring = smem_u32(smem), factor = smem_u32(s_factor), vecs = smem_u32(s_vec);
    bool ok = true;
    int it = 0, piece = 0;  // segments of the run so far
    for (int t = 0; t < tiles && ok; ++t) {
      const int buf = t % S::VEC_BUFS;
      const Tile tile = tile_of<STREAM_ROWS>(list, run, run.lo + t, &segment);
      if (DOWN && tile.starts) ok = mbar_wait_warp(ready, piece & 1, a.check_word, abort_flag);
      if (OUTER && tile.starts && ok) ok = mbar_wait_warp(d2_empty, (piece & 1) ^ 1, a.check_word, abort_flag);
      if (OUTER && ok) ok = mbar_wait_warp(vec_full + 8 * buf, (t / S::VEC_BUFS) & 1, a.check_word, abort_flag);
      if (DOWN && ok) ok = mbar_wait_warp(d1_empty + 8 * (t & 1), ((t >> 1) & 1) ^ 1, a.check_word, abort_flag);
      for (int p = 0; p < pairs && ok; ++p, ++it) {
        const int s = it % SK_STAGES;
        ok = mbar_wait_warp(full + 8 * s, (it / SK_STAGES) & 1, a.check_word, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t stage = ring + s * SK_STAGE;
        if constexpr (DOWN) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 channels each
            umma_f16_ss_if(on, tmem + (t & 1) * RP, umma_desc(stage + k / 4 * SK_TILE + k % 4 * 32),
                           umma_desc(factor + (2 * p + k / 4) * RP * 128 + k % 4 * 32), ID_DOWN, p > 0 || k > 0);
        }
        if constexpr (OUTER) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 rows each
            umma_f16_ss_if(on, tmem + S::COL_OUTER + p * 3 * RP, umma_desc_mn(stage + k * 2048, SK_TILE),
                           umma_desc(vecs + buf * S::VEC + k / 4 * 3 * RP * 128 + k % 4 * 32), ID_OUTER, !tile.starts || k > 0);
        }
        umma_commit_if(on, empty + 8 * s);
      }
      if (!ok) break;
      if (DOWN) umma_commit_if(on, d1_full + 8 * (t & 1));
      if (OUTER) umma_commit_if(on, vec_empty + 8 * buf);
      if (OUTER && tile.ends) umma_commit_if(on, d2_full);
      piece += tile.ends;
    }
  } else if (warp < 4) {
    // ---- operands in, results out.  A tile's vectors go in one tile ahead; behind them its low-rank vectors, and at a segment's end the outer
    // products, come out, so that what the next tile's products overwrite is free.
    if (a.early) pdl_wait();
    pdl_trigger();
    if (tid == 0) abort_flag[PIPE_FRONT] = 0;
    const auto put_factor = [&](int adapter) {
      if (a.by_channel) {  // [channels][rank]: a thread turns one channel's ranks at a time
        for (int c = tid; c < S::CHANNELS; c += SK_SIDE) {
          const uint16_t* f = reinterpret_cast<const uint16_t*>(a.factor) + (static_cast<size_t>(adapter) * a.dim + c0 + c) * a.rank;
          const bool inside = c0 + c < a.dim;
#pragma unroll 16
          for (int r = 0; r < RP; ++r) *reinterpret_cast<uint16_t*>(s_factor + kmajor_at(r, c, RP)) = inside && r < a.rank ? f[r] : 0;
        }
      } else {
#pragma unroll 4
        for (int i = tid; i < RP * S::CHANNELS / 8; i += SK_SIDE) {
          const int r = i / (S::CHANNELS / 8), c = i % (S::CHANNELS / 8) * 8;
          uint4 w = make_uint4(0, 0, 0, 0);
          if (r < a.rank && c0 + c < a.dim) w = *reinterpret_cast<const uint4*>(a.factor + (static_cast<size_t>(adapter) * a.rank + r) * a.dim + c0 + c);
          *reinterpret_cast<uint4*>(s_factor + kmajor_at(r, c, RP)) = w;
        }
      }
      fence_async_proxy();
      mbar_arrive(ready);
    };
    // vectors of tile t: a thread's row, as a column of the operand
    int ahead = segment;
    const auto put_vectors = [&](int t) {
      const Tile tile = tile_of<STREAM_ROWS>(list, run, run.lo + t, &ahead);
      const int buf = t % S::VEC_BUFS, row = s_rows[t * STREAM_ROWS + tid];
      const bool live = row >= 0;
      const float scale = a.scales ? a.scales[ahead] : 1.f;
      const float* v = a.vec + static_cast<size_t>(live ? (a.vec_by_place ? tile.begin + tid : row) : 0) * a.rank;
      float f[RP];
#pragma unroll
      for (int r = 0; r < RP; r += 4) {
        if (a.rank % 4 == 0) {
          const float4 u = live && r < a.rank ? *reinterpret_cast<const float4*>(v + r) : make_float4(0.f, 0.f, 0.f, 0.f);
          f[r] = u.x; f[r + 1] = u.y; f[r + 2] = u.z; f[r + 3] = u.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) f[r + i] = live && r + i < a.rank ? v[r + i] : 0.f;
        }
      }
      if (!mbar_wait_warp(vec_empty + 8 * buf, ((t / S::VEC_BUFS) & 1) ^ 1, a.check_word, abort_flag)) return false;
#pragma unroll
      for (int r = 0; r < RP; r += 2) {
        uint32_t p[3];
        split_pair<3>(scale * f[r], scale * f[r + 1], p);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          char* base = s_vec + buf * S::VEC;
          *reinterpret_cast<uint16_t*>(base + kmajor_at(j * RP + r, tid, 3 * RP)) = static_cast<uint16_t>(p[j] & 0xffffu);
          *reinterpret_cast<uint16_t*>(base + kmajor_at(j * RP + r + 1, tid, 3 * RP)) = static_cast<uint16_t>(p[j] >> 16);
        }
      }
      fence_async_proxy();
      mbar_arrive(vec_full + 8 * buf);
      return true;
    };
    bool ok = true;
    int piece = 0;
    if constexpr (OUTER) ok = put_vectors(0);
    for (int t = 0; t < tiles && ok; ++t) {
      const Tile tile = tile_of<STREAM_ROWS>(list, run, run.lo + t, &segment);
      if constexpr (DOWN) {
        if (tile.starts) put_factor(segment);  // the products of the tiles before are done: their vectors have been taken
      }
      if constexpr (OUTER) {
        if (t + 1 < tiles && S::VEC_BUFS == 2) ok = put_vectors(t + 1);
      }
      if constexpr (DOWN) {
        if (ok) ok = mbar_wait_warp(d1_full + 8 * (t & 1), (t >> 1) & 1, a.check_word, abort_flag);
        if (!ok) break;
        tc_fence_after();
        float* plane = a.planes + (static_cast<size_t>(blockIdx.y) * a.n + tile.begin + tid) * a.rank;
#pragma unroll
        for (int r0 = 0; r0 < RP; r0 += 16) {
          uint32_t w[16];
          __syncwarp();
          tmem_ld16(tmem + (static_cast<uint32_t>(warp * 32) << 16) + (t & 1) * RP + r0, w);
          tmem_ld_wait();
          if (tid < tile.rows) {
            if (a.rank % 4 == 0) {
#pragma unroll
              for (int i = 0; i < 16; i += 4)
                if (r0 + i < a.rank) *reinterpret_cast<uint4*>(plane + r0 + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (r0 + i < a.rank) plane[r0 + i] = __uint_as_float(w[i]);
            }
          }
        }
        tc_fence_before();
        mbar_arrive(d1_empty + 8 * (t & 1));
      }
      if constexpr (OUTER) {
        if (tile.ends) {
          if (ok) ok = mbar_wait_warp(d2_full, piece & 1, a.check_word, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const size_t size = static_cast<size_t>(a.dim) * a.rank;
          const int share = share_of(list, run, segment, blockIdx.x);
          float* out = share < 0 ? a.out + segment * size : a.part + share * size;
          for (int p = 0; p < pairs; ++p) {
            const int c = c0 + p * 128 + tid;
#pragma unroll 1
            for (int r0 = 0; r0 < RP; r0 += 16) {
              uint32_t w[3][16];
              __syncwarp();
              const uint32_t at = tmem + (static_cast<uint32_t>(warp * 32) << 16) + S::COL_OUTER + p * 3 * RP + r0;
#pragma unroll
              for (int j = 0; j < 3; ++j) tmem_ld16(at + j * RP, w[j]);
              tmem_ld_wait();
              if (c >= a.dim) continue;
              float f[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) f[i] = (__uint_as_float(w[2][i]) + __uint_as_float(w[1][i])) + __uint_as_float(w[0][i]);
              if (a.rank_major) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  if (r0 + i < a.rank) out[static_cast<size_t>(r0 + i) * a.dim + c] = f[i];
              } else if (a.rank % 4 == 0) {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                  if (r0 + i < a.rank) *reinterpret_cast<float4*>(out + static_cast<size_t>(c) * a.rank + r0 + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
              } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  if (r0 + i < a.rank) out[static_cast<size_t>(c) * a.rank + r0 + i] = f[i];
              }
            }
          }
          __syncwarp();
          tc_fence_before();
          mbar_arrive(d2_empty);
          ++piece;
        }
        if (t + 1 < tiles && S::VEC_BUFS == 1 && ok) ok = put_vectors(t + 1);
      }
    }
  }
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, S::TMEM);
  }
}

// 16, 32 or 64 threads per place, by the rank.
__global__ void __launch_bounds__(256) lowrank_sum_kernel(SumArgs a) {
  pdl_wait();
  pdl_trigger();
  const int per_cta = a.rank > 32 ? 4 : a.rank > 16 ? 8 : 16, lanes = 256 / per_cta;
  const int place = blockIdx.x * per_cta + threadIdx.x / lanes, r = threadIdx.x % lanes;
  if (place >= a.n || r >= a.rank) return;
  const bool mine = place >= a.off[0] && place < a.off[a.G];
  if (!mine && !a.with_none) return;
  const size_t i = static_cast<size_t>(place) * a.rank + r, plane = static_cast<size_t>(a.n) * a.rank;
  float v = 0.f;
  if (mine) {
#pragma unroll 8
    for (int p = 0; p < a.count; ++p) v += a.planes[p * plane + i];
  }
  a.by_place[i] = v;
  if (a.by_row) a.by_row[static_cast<size_t>(a.perm ? a.perm[place] : place) * a.rank + r] = v;
}

template <int RT>
struct Up {
  static constexpr int ROWS = UP_ROWS, STAGES = 5;
  using Vec = Vectors<RT, 2, ROWS>;
  static constexpr size_t SMEM =
      static_cast<size_t>(LR_WARPS) * STAGES * TILE_BYTES + 2 * Vec::BYTES + sizeof(int) * UP_RUN * ROWS + sizeof(TileList);
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
  TileList& list = *reinterpret_cast<TileList*>(s_rows + UP_RUN * U::ROWS);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  const TileRun run = list_tiles<U::ROWS>(list, a.off, a.segments, a.n, blockIdx.x, a.runs);
  const int tiles = min(run.hi - run.lo, UP_RUN);  // (more only where the segments overlap)
  if (tiles <= 0) {
    pdl_wait();
    pdl_trigger();
    return;
  }
  for (int t = run.lo + warp, s = list.segment; t < run.lo + tiles; t += LR_WARPS) {
    const Tile tile = tile_of<U::ROWS>(list, run, t, &s);
    const int rows = s >= a.G && a.skip_none ? 0 : tile.rows;
    for (int i = lane; i < U::ROWS; i += 32) s_rows[(t - run.lo) * U::ROWS + i] = i < rows ? (a.perm ? a.perm[tile.begin + i] : tile.begin + i) : -1;
  }
  __syncthreads();
  const int c0 = blockIdx.y * UP_CHANNELS + warp * 64;
  Ring<U::STAGES> ring;
  ring.init(smem + warp * U::STAGES * TILE_BYTES, a.base, a.stride, c0, a.base ? a.dim : 0, s_rows, tiles * (U::ROWS / 16));
  if (a.base)
    for (int i = 0; i < U::STAGES - 1; ++i) ring.ask(i);
  int segment = list.segment, ahead = segment;
  uint32_t up[RT][2][4][2];  // [16 ranks][32 channels][8 of them][k half]
  const auto load_factor = [&](int adapter) {
#pragma unroll
    for (int s = 0; s < RT; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int r = 16 * s + 8 * half + 2 * q, c8 = c0 + 32 * h + 8 * (g >> 1);  // two ranks, eight channels
          if (adapter >= a.G) {
#pragma unroll
            for (int i = 0; i < 4; ++i) up[s][h][i][half] = 0;
          } else if (a.by_rank) {
            const __nv_bfloat16* f = a.factor + static_cast<size_t>(adapter) * a.rank * a.dim;
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
            const uint16_t* f = reinterpret_cast<const uint16_t*>(a.factor) + static_cast<size_t>(adapter) * a.rank * a.dim;
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
  };
  load_factor(segment);
  pdl_wait();
  pdl_trigger();
  Vec vec;
  float scale = 1.f;
  const auto ask_vectors = [&](int t) {
    if (t >= tiles) return;
    const Tile tile = tile_of<U::ROWS>(list, run, run.lo + t, &ahead);
    const bool none = ahead >= a.G;
    scale = a.scales && !none ? a.scales[ahead] : 1.f;
    vec.ask(a.vec, a.rank, 0, none ? 0 : tile.rows, [&](int i) { return tile.begin + i; });
  };
  ask_vectors(0);
  vec.put(s_vec, scale);
  for (int t = 0, buf = 0; t < tiles; ++t, buf ^= 1) {
    __syncthreads();  // the vectors of these rows are there
    ask_vectors(t + 1);
    if (t > 0 && tile_of<U::ROWS>(list, run, run.lo + t, &segment).starts) load_factor(segment);
    const uint32_t vecs = smem_addr(s_vec + buf * Vec::BYTES);
#pragma unroll 1
    for (int k = 0; k < U::ROWS / 16; ++k) {
      const int stage = t * (U::ROWS / 16) + k;
      uint32_t tile = 0;
      if (a.base) {
        tile = ring.get(stage);
        ring.ask(stage + U::STAGES - 1);
      }
      if (s_rows[stage * 16] < 0) continue;
      float d[2][4][4];
#pragma unroll
      for (int s = 0; s < RT; ++s)
#pragma unroll
        for (int p = 1; p >= 0; --p) {
          uint32_t vf[4];
          ldmatrix4(vf, vecs + (p * U::ROWS + k * 16 + (lane & 7) + (lane >> 3 & 1) * 8) * Vec::V_BYTES + (2 * s + (lane >> 4)) * 16);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (s == 0 && p == 1) mma_bf16_first(d[h][i], vf, up[s][h][i][0], up[s][h][i][1]);
              else mma_bf16(d[h][i], vf, up[s][h][i][0], up[s][h][i][1]);
            }
        }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int row = g + 8 * half, at = s_rows[stage * 16 + row];
        if (at < 0) continue;
        __nv_bfloat16* y = a.out + static_cast<size_t>(at) * a.stride;
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
cudaError_t launch_stream_of(const StreamArgs& a, cudaStream_t st) {
  constexpr size_t smem = Stream<RT>::smem(DOWN, OUTER);
  const cudaError_t e = allow_smem<lowrank_stream_kernel<RT, DOWN, OUTER>>(static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_chain(lowrank_stream_kernel<RT, DOWN, OUTER>, dim3(a.runs, (a.dim + Stream<RT>::CHANNELS - 1) / Stream<RT>::CHANNELS), dim3(SK_THREADS), smem,
                      st, a);
}

template <int RT>
cudaError_t launch_stream_rank(const StreamArgs& a, cudaStream_t st) {
  if (a.factor && a.vec) return launch_stream_of<RT, true, true>(a, st);
  return a.factor ? launch_stream_of<RT, true, false>(a, st) : launch_stream_of<RT, false, true>(a, st);
}

template <int RT>
cudaError_t launch_up_rank(const UpArgs& a, cudaStream_t st) {
  const cudaError_t e = allow_smem<lowrank_up_kernel<RT>>(static_cast<int>(Up<RT>::SMEM));
  if (e != cudaSuccess) return e;
  return launch_chain(lowrank_up_kernel<RT>, dim3(a.runs, (a.dim + UP_CHANNELS - 1) / UP_CHANNELS), dim3(LR_THREADS), Up<RT>::SMEM, st, a);
}

}  // namespace

cudaError_t launch_lowrank_stream(const StreamArgs& a, cudaStream_t st) {
  if (a.rank <= 16) return launch_stream_rank<1>(a, st);
  return a.rank <= 32 ? launch_stream_rank<2>(a, st) : launch_stream_rank<4>(a, st);
}

cudaError_t launch_lowrank_sum(const SumArgs& a, cudaStream_t st) {
  const int per_cta = a.rank > 32 ? 4 : a.rank > 16 ? 8 : 16;
  return launch_chain(lowrank_sum_kernel, dim3((a.n + per_cta - 1) / per_cta), dim3(256), 0, st, a);
}

cudaError_t launch_lowrank_up(const UpArgs& a, cudaStream_t st) {
  if (a.rank <= 16) return launch_up_rank<1>(a, st);
  return a.rank <= 32 ? launch_up_rank<2>(a, st) : launch_up_rank<4>(a, st);
}

}  // namespace emoe

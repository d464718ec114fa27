// Low-rank adapters on many bf16 rows.  Three kernels that each read their activations once:
//   stream  x (dy) goes by: shares of the low-rank vectors v = A x (B^T dy), and in the backward pass, from the same
//           tiles, the outer products with the vectors of the other side, dB = s sum dy v^T (dA = sum dv x^T)
//   sum     the shares of the vectors, one per 512 channels, added in order
//   up      y = base + s B v (dx = dx_base + A^T s dv)
// A value of x takes part in 16 to 64 multiply-adds of v and three times as many of the outer products, too much for the instructions
// that registers feed once the rank is 32 or 64, and any instruction that a thread spends on a value shows: so the rows go from cp.async
// (they may stand in any order) to tcgen05, and what comes out of tensor memory is small, or meets base on its way out.
// A CTA owns 512 (256) channels of an even run of the rows.
#include "lowrank.cuh"
#include "pipe.cuh"
#include "umma.cuh"

namespace emoe {
namespace {

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool live) {
  const int bytes = live ? 16 : 0;  // none: the place is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// byte of value `k` of row `n` in swizzled tiles of 64 values, `rows` rows each
__device__ __forceinline__ uint32_t tile_at(int n, int k, int rows) {
  return k / 64 * rows * 128 + n * 128 + ((k % 64 / 8 ^ (n & 7)) << 4) + k % 8 * 2;
}

constexpr int SIDE = 128;  // threads of a role that moves data
constexpr int TILE = STREAM_ROWS * 128, STAGE = 2 * TILE;  // 128 rows x 64 values; a stage: 128 channels

// the barrier receives an arrival once all copies that this thread has asked for so far are there
__device__ __forceinline__ void copy_arrive(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }

// Copies the rows of a run, 128 channels at a time, into a ring of stages.  A thread copies 16 bytes of every eighth row of a tile; places
// without a row and channels beyond the end become zeros (as does all that is not wanted).  FOR_MMA: the tensor cores read the
// stage, so that the thread itself sees its copies land, fences them and arrives, before it waits for the next free stage (behind that wait
// the products of a stage would not start before those in front of it are done: 14 instead of 10 us per 67 MB).  Else threads read it
// and the copies arrive by themselves.
template <int STAGES, bool FOR_MMA>
__device__ __forceinline__ void copy_rows(const __nv_bfloat16* act, bool wanted, size_t stride, int dim, int c0, int pairs, RunWalk<STREAM_ROWS> walk, const int* s_rows,
                                          uint32_t ring, uint32_t full, uint32_t empty, int thread, int* check_word, volatile int* abort_flag) {
  const int piece = thread & 15, row0 = thread >> 4;
  const uint32_t dst = ring + (piece >> 3) * TILE + row0 * 128 + (((piece & 7) ^ row0) << 4);
  const __nv_bfloat16* row[STREAM_ROWS / 8];
  int it = 0;
  bool ok = true;
  const auto landed = [&](int stage) {
    fence_async_proxy();
    mbar_arrive(full + 8 * (stage % STAGES));
  };
  while (walk.more() && ok) {
    walk.next();
    uint32_t live = 0;
#pragma unroll
    for (int j = 0; j < STREAM_ROWS / 8; ++j) {
      const int r = s_rows[(walk.at - 1 - walk.lo) * STREAM_ROWS + row0 + 8 * j];
      if (r >= 0 && wanted) live |= 1u << j;
      row[j] = act + static_cast<size_t>(max(r, 0)) * stride;
    }
    for (int p = 0; p < pairs; ++p, ++it) {
      const int s = it % STAGES, c = c0 + p * 128 + piece * 8;
      if constexpr (FOR_MMA) {
        copy_wait<STAGES - 2>();
        if (it >= STAGES - 1) landed(it - (STAGES - 1));
      }
      ok = mbar_wait(empty + 8 * s, ((it / STAGES) & 1) ^ 1, check_word, abort_flag);
      if (!ok) break;
      const bool inside = c < dim;
#pragma unroll
      for (int j = 0; j < STREAM_ROWS / 8; ++j) copy_async16(dst + s * STAGE + j * 1024, row[j] + (inside ? c : 0), inside && (live >> j & 1u));
      if constexpr (FOR_MMA) copy_commit();
      else copy_arrive(full + 8 * s);
    }
  }
  copy_commit();
  copy_wait<0>();
  if (FOR_MMA && ok)
    for (int s = max(0, it - (STAGES - 1)); s < it; ++s) landed(s);
}

// A factor of `channels` channels from c0 on as tiles [rank][64 channels].  by_channel: it is stored [dim][rank], and a thread turns one
// channel's ranks; else [rank][dim].  Channels and ranks beyond the end are zeros.  SIDE threads.
template <int RP, int CHANNELS>
__device__ __forceinline__ void put_factor(char* tiles, const __nv_bfloat16* factor, bool by_channel, int adapter, int dim, int rank, int c0, int thread) {
  if (by_channel) {
    const uint16_t* f = reinterpret_cast<const uint16_t*>(factor) + (static_cast<size_t>(adapter) * dim + c0) * rank;
    constexpr int N = CHANNELS / SIDE, W = RP < 32 ? 2 : 4;  // channels of a thread, words of eight ranks asked for together
    if (rank % 8 == 0) {
#pragma unroll 1
      for (int r0 = 0; r0 < RP; r0 += 8 * W) {
        uint4 w[N][W];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int h = 0; h < W; ++h) {
            const int c = thread + j * SIDE;
            w[j][h] = c0 + c < dim && r0 + 8 * h < rank ? *reinterpret_cast<const uint4*>(f + static_cast<size_t>(c) * rank + r0 + 8 * h) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int h = 0; h < W; ++h) {
            const uint32_t v[4] = {w[j][h].x, w[j][h].y, w[j][h].z, w[j][h].w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<uint16_t*>(tiles + tile_at(r0 + 8 * h + i, thread + j * SIDE, RP)) = static_cast<uint16_t>(v[i / 2] >> (16 * (i % 2)));
          }
      }
    } else {
      for (int c = thread; c < CHANNELS; c += SIDE) {
        const bool inside = c0 + c < dim;
#pragma unroll 16
        for (int r = 0; r < RP; ++r)
          *reinterpret_cast<uint16_t*>(tiles + tile_at(r, c, RP)) = inside && r < rank ? f[static_cast<size_t>(c) * rank + r] : 0;
      }
    }
  } else {
#pragma unroll 8
    for (int i = thread; i < RP * CHANNELS / 8; i += SIDE) {
      const int r = i / (CHANNELS / 8), c = i % (CHANNELS / 8) * 8;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r < rank && c0 + c < dim) w = *reinterpret_cast<const uint4*>(factor + (static_cast<size_t>(adapter) * rank + r) * dim + c0 + c);
      *reinterpret_cast<uint4*>(tiles + tile_at(r, c, RP)) = w;
    }
  }
}

// N values of a low-rank vector, zeros from `count` on; words: vectors are whole 16-byte words
template <int N>
__device__ __forceinline__ void load_vector(const float* v, int count, bool words, bool live, float (&f)[N]) {
#pragma unroll
  for (int r = 0; r < N; r += 4) {
    if (words) {
      const float4 u = live && r < count ? *reinterpret_cast<const float4*>(v + r) : make_float4(0.f, 0.f, 0.f, 0.f);
      f[r] = u.x; f[r + 1] = u.y; f[r + 2] = u.z; f[r + 3] = u.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[r + i] = live && r + i < count ? v[r + i] : 0.f;
    }
  }
}

constexpr uint32_t BF16_F32 = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);  // instruction descriptor: bf16 x bf16 -> fp32, M = 128
__host__ __device__ constexpr uint32_t columns(int n) { return static_cast<uint32_t>(n / 8) << 17; }
constexpr uint32_t A_BY_COLUMNS = 1u << 15, B_BY_COLUMNS = 1u << 16;  // operand is MN-major

// ---- stream -------------------------------------------------------------------------------------

// Roles: warps 0-3 bring the factor and the vectors into shared memory as operands and carry results out of tensor memory, warps 4-7
// copy the rows, warp 8 issues the products.
constexpr int SK_THREADS = 288, SK_STAGES = 4;

template <int RT>
struct Stream {
  static constexpr int RP = RT * 16, CHANNELS = stream_channels(RP), PAIRS = CHANNELS / 128;
  static constexpr int FACTOR = CHANNELS / 64 * RP * 128;      // [rank][channels], K-major tiles of 64 channels
  static constexpr int VEC = (3 * RP + 63) / 64 * TILE;        // [128 rows][three parts of rank], tiles of 64 values
  __host__ __device__ static constexpr int vec_bufs(bool down) { return RT == 4 || (RT == 2 && down) ? 1 : 2; }
  static constexpr int COL_OUTER = 2 * RP, COLS = COL_OUTER + PAIRS * 3 * RP, TMEM = COLS <= 256 ? 256 : 512;
  static_assert(COLS <= 512, "tensor memory has 512 columns");
  // two factors where there is room: the next segment's comes in ahead (a change of segments stops the products for some 3 us else)
  __host__ __device__ static constexpr int factor_bufs(bool outer) { return RT == 1 || !outer ? 2 : 1; }
  static constexpr size_t smem(bool down, bool outer) {
    return 1024 + static_cast<size_t>(SK_STAGES) * STAGE + (down ? factor_bufs(outer) * FACTOR : 0) + (outer ? vec_bufs(down) * VEC : 0) + sizeof(int) * STREAM_RUN * STREAM_ROWS + sizeof(TileList);
  }
};

// The products, for a tile X of 128 rows x 128 channels (two swizzled tiles of 64, as cp.async leaves them):
//   vectors [128 rows][rank]              += X F^T          X read along its rows (K-major), 16 channels per instruction
//   outer   [128 channels][3 x rank]      += X^T V          X read along its columns (MN-major), 16 rows per instruction
// V are the rows' vectors in three bf16 parts side by side, so that the three products cost one instruction; they are added at the
// end.  Both sums stay in tensor memory: the vectors over the CTA's channels, the outer products over the rows of a segment in its run.  The
// tensor cores cut what they add, so a run is no longer than 1024 rows: the vectors are off by 5e-7 of their norm over 512 channels and 2.4e-7 over
// 256, dB by 1e-7 over 100 rows and 2.6e-7 over runs of 1024, dA (with its vectors' own error) by 1.5e-7 to 7e-7.  Rounded sums have 1e-7 to 2e-7.
template <int RT, bool DOWN, bool OUTER>
__global__ void __launch_bounds__(SK_THREADS, 1) lowrank_stream_kernel(StreamArgs a) {
  using S = Stream<RT>;
  constexpr int RP = S::RP, PAIRS = S::PAIRS, VEC_BUFS = S::vec_bufs(DOWN), FACTOR_BUFS = S::factor_bufs(OUTER);
  extern __shared__ char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * SK_STAGES + 12];  // full, empty: stages; ready: factors
  __shared__ uint32_t tmem_slot;
  __shared__ int wait_words[PIPE_WORDS];
  volatile int* abort_flag = wait_words + PIPE_ABORT;
  char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  char* s_factor = smem + SK_STAGES * STAGE;
  char* s_vec = s_factor + (DOWN ? FACTOR_BUFS * S::FACTOR : 0);
  int* s_rows = reinterpret_cast<int*>(s_vec + (OUTER ? VEC_BUFS * S::VEC : 0));
  TileList& list = *reinterpret_cast<TileList*>(s_rows + STREAM_RUN * STREAM_ROWS);
  const uint32_t full = smem_u32(bars), empty = full + 8 * SK_STAGES, d1_full = empty + 8 * SK_STAGES, d1_empty = d1_full + 16,
                 vec_full = d1_empty + 16, vec_empty = vec_full + 16, ready = vec_empty + 16, d2_full = ready + 16, d2_empty = d2_full + 8;
  const int tid = threadIdx.x, warp = uniform_warp();
  if (tid == 0) {
    for (int i = 0; i < SK_STAGES; ++i) {
      mbar_init(full + 8 * i, SIDE);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(d1_full + 8 * i, 1);
      mbar_init(d1_empty + 8 * i, SIDE);
      mbar_init(vec_full + 8 * i, SIDE);
      mbar_init(vec_empty + 8 * i, 1);
      mbar_init(ready + 8 * i, SIDE);
    }
    mbar_init(d2_full, 1);
    mbar_init(d2_empty, SIDE);
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
  list_rows<STREAM_ROWS>(list, run, a.perm, a.G, true, s_rows);
  if (warp == 8) tmem_alloc(smem_u32(&tmem_slot), S::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int c0 = blockIdx.y * S::CHANNELS;
  const int pairs = min(PAIRS, (a.dim - c0 + 127) / 128);  // of 128 channels; what the last has too many reads as zeros
  RunWalk<STREAM_ROWS> walk(list, run);

  if (warp >= 4 && warp < 8) {
    // ---- rows
    copy_rows<SK_STAGES, true>(a.act, true, a.stride, a.dim, c0, pairs, walk, s_rows, smem_u32(smem), full, empty, tid - 128, a.check_word, abort_flag);
  } else if (warp == 8) {
    // ---- products
    const uint32_t on = elect_one();
    constexpr uint32_t ID_DOWN = BF16_F32 | columns(RP), ID_OUTER = BF16_F32 | A_BY_COLUMNS | B_BY_COLUMNS | columns(3 * RP);
    const uint32_t ring = smem_u32(smem), factor = smem_u32(s_factor), vecs = smem_u32(s_vec);
    bool ok = true;
    int it = 0, piece = 0;  // segments of the run so far
    for (int t = 0; walk.more() && ok; ++t) {
      const int buf = t % VEC_BUFS;
      const Tile tile = walk.next();
      if (DOWN && tile.starts) ok = mbar_wait_warp(ready + 8 * (piece & 1), (piece >> 1) & 1, a.check_word, abort_flag);
      if (OUTER && tile.starts && ok) ok = mbar_wait_warp(d2_empty, (piece & 1) ^ 1, a.check_word, abort_flag);
      if (OUTER && ok) ok = mbar_wait_warp(vec_full + 8 * buf, (t / VEC_BUFS) & 1, a.check_word, abort_flag);
      if (DOWN && ok) ok = mbar_wait_warp(d1_empty + 8 * (t & 1), ((t >> 1) & 1) ^ 1, a.check_word, abort_flag);
      for (int p = 0; p < pairs && ok; ++p, ++it) {
        const int s = it % SK_STAGES;
        ok = mbar_wait_warp(full + 8 * s, (it / SK_STAGES) & 1, a.check_word, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t stage = ring + s * STAGE;
        if constexpr (DOWN) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 channels each
            umma_f16_ss_if(on, tmem + (t & 1) * RP, umma_desc(stage + k / 4 * TILE + k % 4 * 32),
                           umma_desc(factor + piece % FACTOR_BUFS * S::FACTOR + (2 * p + k / 4) * RP * 128 + k % 4 * 32), ID_DOWN, p > 0 || k > 0);
        }
        if constexpr (OUTER) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // 16 rows each
            umma_f16_ss_if(on, tmem + S::COL_OUTER + p * 3 * RP, umma_desc_mn(stage + k * 2048, TILE),
                           umma_desc_mn(vecs + buf * S::VEC + k * 2048, TILE), ID_OUTER, !tile.starts || k > 0);
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
    // the vector of a thread's row of the next tile: asked for and cut into parts ahead, put down once its place is free
    RunWalk<STREAM_ROWS> ahead = walk;
    int next = 0;
    float f[RP];
    float scale = 1.f;
    const auto ask_vectors = [&] {
      const Tile tile = ahead.next();
      const bool live = tid < tile.rows;
      scale = a.scales ? a.scales[ahead.segment] : 1.f;
      load_vector<RP>(a.vec + static_cast<size_t>(!live ? 0 : a.vec_by_place ? tile.begin + tid : s_rows[(ahead.at - 1 - run.lo) * STREAM_ROWS + tid]) * a.rank, a.rank, a.rank % 4 == 0, live, f);
    };
    const auto put_vectors = [&] {
      const int buf = next % VEC_BUFS;
      uint32_t part[3][RP / 2];
#pragma unroll
      for (int r = 0; r < RP; r += 2) {
        uint32_t p[3];
        split_pair<3>(scale * f[r], scale * f[r + 1], p);
#pragma unroll
        for (int j = 0; j < 3; ++j) part[j][r / 2] = p[j];
      }
      if (!mbar_wait_warp(vec_empty + 8 * buf, ((next / VEC_BUFS) & 1) ^ 1, a.check_word, abort_flag)) return false;
#pragma unroll
      for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int r = 0; r < RP; r += 8)
          *reinterpret_cast<uint4*>(s_vec + buf * S::VEC + tile_at(tid, j * RP + r, STREAM_ROWS)) =
              make_uint4(part[j][r / 2], part[j][r / 2 + 1], part[j][r / 2 + 2], part[j][r / 2 + 3]);
      fence_async_proxy();
      mbar_arrive(vec_full + 8 * buf);
      ++next;
      return true;
    };
    int factors = 0;
    const auto bring_factor = [&](int adapter) {
      put_factor<RP, S::CHANNELS>(s_factor + factors % FACTOR_BUFS * S::FACTOR, a.factor, a.by_channel, adapter, a.dim, a.rank, c0, tid);
      fence_async_proxy();
      mbar_arrive(ready + 8 * (factors & 1));
      ++factors;
    };
    bool ok = true;
    int piece = 0;
    if constexpr (DOWN && FACTOR_BUFS == 2) bring_factor(walk.segment);
    if constexpr (OUTER) {
      ask_vectors();
      ok = put_vectors();
    }
    for (int t = 0; walk.more() && ok; ++t) {
      const Tile tile = walk.next();
      bool asked = false;
      if constexpr (DOWN) {
        // (the products of the tiles before are done: their vectors have been taken)
        if (FACTOR_BUFS == 1 && tile.starts) bring_factor(walk.segment);
        if (FACTOR_BUFS == 2 && tile.ends && walk.more()) bring_factor(walk.next_segment());
      }
      if constexpr (OUTER) {
        asked = ahead.more();
        if (asked) ask_vectors();
        if (asked && VEC_BUFS == 2) ok = put_vectors();
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
          const int share = share_of(list, run, walk.segment, blockIdx.x);
          float* out = share < 0 ? a.out + walk.segment * size : a.part + share * size;
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
        if (asked && VEC_BUFS == 1 && ok) ok = put_vectors();
      }
    }
  }
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, S::TMEM);
  }
}

// A thread adds four neighbouring ranks of a place.
__global__ void __launch_bounds__(256) lowrank_sum_kernel(SumArgs a) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0) check_offsets(a.off, a.G, a.n, a.check_word);
  const int lanes = a.rank > 32 ? 16 : a.rank > 16 ? 8 : 4, place = blockIdx.x * (256 / lanes) + threadIdx.x / lanes, r = threadIdx.x % lanes * 4;
  if (place >= a.n || r >= a.rank) return;
  const bool mine = place >= a.off[0] && place < a.off[a.G];
  if (!mine && !a.with_none) return;
  const size_t i = static_cast<size_t>(place) * a.rank + r, plane = static_cast<size_t>(a.n) * a.rank;
  const size_t row = a.by_row ? static_cast<size_t>(a.perm ? a.perm[place] : place) * a.rank + r : 0;
  if (a.rank % 4 == 0) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (mine) {
#pragma unroll 8
      for (int p = 0; p < a.count; ++p) {
        const float4 u = *reinterpret_cast<const float4*>(a.planes + p * plane + i);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
      }
    }
    *reinterpret_cast<float4*>(a.by_place + i) = v;
    if (a.by_row) *reinterpret_cast<float4*>(a.by_row + row) = v;
  } else {
    for (int k = 0; k < 4 && r + k < a.rank; ++k) {
      float v = 0.f;
      if (mine)
        for (int p = 0; p < a.count; ++p) v += a.planes[p * plane + i + k];
      a.by_place[i + k] = v;
      if (a.by_row) a.by_row[row + k] = v;
    }
  }
}

// ---- up -----------------------------------------------------------------------------------------

// Roles: warps 0-7 add base and write, eight to a stage (a stage is held while they do: with four, and two sets of them, 1.6 us a stage
// whatever its rows), 8-11 copy base, 12 issues the products, 13-16
// bring factor and vectors.
constexpr int UP_THREADS = 544, UP_ACC = 4;  // accumulators of 128 rows x 128 channels: all of tensor memory

template <int RT>
struct Up {
  static constexpr int RP = RT * 16, CHANNELS = stream_channels(RP), STAGES = RT == 4 ? 3 : 4;
  static constexpr int FACTOR = CHANNELS / 64 * RP * 128;            // [rank][channels], tiles of 64 channels; two of them
  static constexpr int VEC = (2 * RP + 63) / 64 * STREAM_ROWS * 128;  // [128 rows][two parts of rank], K-major tiles of 64 values
  static constexpr int VEC_BUFS = RT == 1 ? 2 : 1;
  static constexpr size_t SMEM =
      1024 + static_cast<size_t>(STAGES) * STAGE + 2 * FACTOR + VEC_BUFS * VEC + sizeof(int) * UP_RUN * STREAM_ROWS + sizeof(TileList);
};

// y = base + s B v: the product V F of the rows' vectors (two bf16 parts, rows of the A operand) with the factor's tiles read along their
// columns comes out of tensor memory, a row per lane.  Base stands in its stage as it was copied, swizzled, so that a lane reads its
// row's pieces without bank conflicts; the rounded sum goes back to the same place, and the warp writes its 32 rows from there in whole 128-byte
// lines.  (Base through the tensor cores, as a product with ones on a diagonal, would save the additions, but a NaN in one row would
// reach the others of its tile.)
template <int RT>
__global__ void __launch_bounds__(UP_THREADS, 1) lowrank_up_kernel(UpArgs a) {
  using U = Up<RT>;
  constexpr int RP = U::RP;
  extern __shared__ char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * U::STAGES + 2 * UP_ACC + 8];
  __shared__ uint32_t tmem_slot;
  __shared__ int wait_words[PIPE_WORDS];
  volatile int* abort_flag = wait_words + PIPE_ABORT;
  char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  char* s_factor = smem + U::STAGES * STAGE;
  char* s_vec = s_factor + 2 * U::FACTOR;
  int* s_rows = reinterpret_cast<int*>(s_vec + U::VEC_BUFS * U::VEC);
  TileList& list = *reinterpret_cast<TileList*>(s_rows + UP_RUN * STREAM_ROWS);
  const uint32_t full = smem_u32(bars), empty = full + 8 * U::STAGES, acc_full = empty + 8 * U::STAGES, acc_empty = acc_full + 8 * UP_ACC,
                 vec_full = acc_empty + 8 * UP_ACC, vec_empty = vec_full + 16, ready = vec_empty + 16, factor_free = ready + 16;
  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < U::STAGES; ++i) {
      mbar_init(full + 8 * i, SIDE);
      mbar_init(empty + 8 * i, 2 * SIDE);
    }
    for (int i = 0; i < UP_ACC; ++i) {
      mbar_init(acc_full + 8 * i, 1);
      mbar_init(acc_empty + 8 * i, 2 * SIDE);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(vec_full + 8 * i, SIDE);
      mbar_init(vec_empty + 8 * i, 1);
      mbar_init(ready + 8 * i, SIDE);
      mbar_init(factor_free + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    wait_words[PIPE_ABORT] = 0;
    wait_words[PIPE_FRONT] = 1;  // until the vectors' warps are past their wait for the kernel in front
  }
  TileRun run = list_tiles<STREAM_ROWS>(list, a.off, a.segments, a.n, blockIdx.x, a.runs);
  run.hi = min(run.hi, run.lo + UP_RUN);  // (longer only where the segments overlap, which the kernel in front has reported)
  if (run.lo >= run.hi) {
    pdl_wait();
    pdl_trigger();
    return;
  }
  list_rows<STREAM_ROWS>(list, run, a.perm, a.G, !a.skip_none, s_rows);
  if (warp == 12) tmem_alloc(smem_u32(&tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int c0 = blockIdx.y * U::CHANNELS, pairs = min(U::CHANNELS / 128, (a.dim - c0 + 127) / 128);
  RunWalk<STREAM_ROWS> walk(list, run);

  if (warp < 8) {
    const int h = warp >> 2, r0 = (warp & 3) * 32, own = r0 + lane;  // the warp's 64 channels and rows; the lane's row
    bool ok = true;
    int it = 0;
    bool waited = false;
    while (walk.more() && ok) {
      walk.next();
      const int* rows = s_rows + (walk.at - 1 - run.lo) * STREAM_ROWS;
      const bool any = rows[r0] >= 0;  // (those with a row come first)
      for (int p = 0; p < pairs; ++p, ++it) {
        const int s = it % U::STAGES, b = it % UP_ACC;
        ok = mbar_wait_warp(full + 8 * s, (it / U::STAGES) & 1, a.check_word, abort_flag) &&
             mbar_wait_warp(acc_full + 8 * b, (it / UP_ACC) & 1, a.check_word, abort_flag);
        if (!ok) break;
        if (!waited) {  // what is written may be what the kernels in front read
          pdl_wait();
          waited = true;
        }
        tc_fence_after();
        char* stage = smem + s * STAGE;
        if (any) {
#pragma unroll
          for (int q = 2 * h; q < 2 * h + 2; ++q) {  // 32 channels each
            uint32_t w[32];
            tmem_ld32(tmem + (static_cast<uint32_t>(r0) << 16) + b * 128 + q * 32, w);
            uint4 u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const uint4*>(stage + tile_at(own, q * 32 + i * 8, STREAM_ROWS));
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              Piece<__nv_bfloat16, 8> piece = {{u[i].x, u[i].y, u[i].z, u[i].w}};
              float f[8];
              widen<__nv_bfloat16, 8>(piece, f);
#pragma unroll
              for (int j = 0; j < 8; ++j) f[j] += __uint_as_float(w[i * 8 + j]);
              piece = narrow<__nv_bfloat16, 8>(f);
              *reinterpret_cast<uint4*>(stage + tile_at(own, q * 32 + i * 8, STREAM_ROWS)) = make_uint4(piece.w[0], piece.w[1], piece.w[2], piece.w[3]);
            }
          }
          __syncwarp();
          const int c = c0 + p * 128 + h * 64 + (lane & 7) * 8;
          if (c < a.dim) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int r = r0 + (lane >> 3) + 4 * j, at = rows[r];
              const uint4 u = *reinterpret_cast<const uint4*>(stage + tile_at(r, h * 64 + (lane & 7) * 8, STREAM_ROWS));
              if (at >= 0) *reinterpret_cast<uint4*>(a.out + static_cast<size_t>(at) * a.stride + c) = u;
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        mbar_arrive(acc_empty + 8 * b);
        mbar_arrive(empty + 8 * s);
      }
    }
  } else if (warp < 12) {
    copy_rows<U::STAGES, false>(a.base ? a.base : a.out, a.base != nullptr, a.stride, a.dim, c0, pairs, walk, s_rows, smem_u32(smem), full, empty,
                                tid - 256, a.check_word, abort_flag);
  } else if (warp == 12) {
    const uint32_t on = elect_one();
    const uint32_t factor = smem_u32(s_factor), vecs = smem_u32(s_vec);
    bool ok = true;
    int it = 0, piece = 0;
    for (int t = 0; walk.more() && ok; ++t) {
      const int buf = t % U::VEC_BUFS;
      const Tile tile = walk.next();
      if (tile.starts) ok = mbar_wait_warp(ready + 8 * (piece & 1), (piece >> 1) & 1, a.check_word, abort_flag);
      if (ok) ok = mbar_wait_warp(vec_full + 8 * buf, (t / U::VEC_BUFS) & 1, a.check_word, abort_flag);
      for (int p = 0; p < pairs && ok; ++p, ++it) {
        const int b = it % UP_ACC;
        ok = mbar_wait_warp(acc_empty + 8 * b, ((it / UP_ACC) & 1) ^ 1, a.check_word, abort_flag);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int part = 1; part >= 0; --part)
#pragma unroll
          for (int k = 0; k < RT; ++k) {  // 16 ranks each
            const int at = part * RP + k * 16;
            umma_f16_ss_if(on, tmem + b * 128, umma_desc(vecs + buf * U::VEC + at / 64 * TILE + at % 64 * 2),
                           umma_desc_mn(factor + (piece & 1) * U::FACTOR + 2 * p * RP * 128 + k * 2048, RP * 128), BF16_F32 | B_BY_COLUMNS | columns(128), part == 0 || k > 0);
          }
        umma_commit_if(on, acc_full + 8 * b);
      }
      if (!ok) break;
      umma_commit_if(on, vec_empty + 8 * buf);
      if (tile.ends) umma_commit_if(on, factor_free + 8 * (piece & 1));
      piece += tile.ends;
    }
  } else {
    const int thread = tid - 13 * 32;
    bool ok = true;
    int piece = 0;
    for (int t = 0; walk.more() && ok; ++t) {
      const Tile tile = walk.next();
      const bool none = walk.segment >= a.G;
      if (tile.starts) {  // ahead of the products of the segment in front
        ok = mbar_wait_warp(factor_free + 8 * (piece & 1), ((piece >> 1) & 1) ^ 1, a.check_word, abort_flag);
        if (!ok) break;
        // the rows of no adapter: a factor of zeros
        put_factor<RP, U::CHANNELS>(s_factor + (piece & 1) * U::FACTOR, a.factor, !a.by_rank, none ? 0 : walk.segment, none ? 0 : a.dim, a.rank, c0,
                                          thread);
        fence_async_proxy();
        mbar_arrive(ready + 8 * (piece & 1));
        ++piece;
      }
      if (t == 0) {
        pdl_wait();
        pdl_trigger();
        if (thread == 0) abort_flag[PIPE_FRONT] = 0;
      }
      const int buf = t % U::VEC_BUFS;
      const float scale = a.scales && !none ? a.scales[walk.segment] : 1.f;
      const bool live = !none && thread < tile.rows;
      float f[RP];
      load_vector<RP>(a.vec + static_cast<size_t>(live ? tile.begin + thread : 0) * a.rank, a.rank, a.rank % 4 == 0, live, f);
      ok = mbar_wait_warp(vec_empty + 8 * buf, ((t / U::VEC_BUFS) & 1) ^ 1, a.check_word, abort_flag);
      if (!ok) break;
#pragma unroll
      for (int r = 0; r < RP; r += 8) {
        uint32_t w[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t part[2];
          split_pair<2>(scale * f[r + 2 * i], scale * f[r + 2 * i + 1], part);
          w[0][i] = part[0];
          w[1][i] = part[1];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
          *reinterpret_cast<uint4*>(s_vec + buf * U::VEC + tile_at(thread, j * RP + r, STREAM_ROWS)) = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
      }
      fence_async_proxy();
      mbar_arrive(vec_full + 8 * buf);
    }
  }
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
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
  return launch_chain(lowrank_up_kernel<RT>, dim3(a.runs, (a.dim + Up<RT>::CHANNELS - 1) / Up<RT>::CHANNELS), dim3(UP_THREADS),
                      Up<RT>::SMEM, st, a);
}

}  // namespace

cudaError_t launch_lowrank_stream(const StreamArgs& a, cudaStream_t st) {
  if (a.rank <= 16) return launch_stream_rank<1>(a, st);
  return a.rank <= 32 ? launch_stream_rank<2>(a, st) : launch_stream_rank<4>(a, st);
}

cudaError_t launch_lowrank_sum(const SumArgs& a, cudaStream_t st) {
  const int per_cta = a.rank > 32 ? 16 : a.rank > 16 ? 32 : 64;
  return launch_chain(lowrank_sum_kernel, dim3((a.n + per_cta - 1) / per_cta), dim3(256), 0, st, a);
}

cudaError_t launch_lowrank_up(const UpArgs& a, cudaStream_t st) {
  if (a.rank <= 16) return launch_up_rank<1>(a, st);
  return a.rank <= 32 ? launch_up_rank<2>(a, st) : launch_up_rank<4>(a, st);
}

}  // namespace emoe

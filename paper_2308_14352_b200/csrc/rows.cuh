// Rows of activations as the operators for training and adapters move them: a piece is VEC consecutive values of one
// row, loaded as one or two wide words and widened to fp32 registers.  Also the host-side pieces that their entry points share.
#pragma once
#include "common.cuh"

namespace emoe {

// VEC values of T as 32-bit words; a piece of one 16-bit value sits in the low half of its word.
template <typename T, int VEC>
struct Piece {
  static constexpr int WORDS = (VEC * static_cast<int>(sizeof(T)) + 3) / 4;
  uint32_t w[WORDS];
};

// Reads that are used once (activations): not kept in L1.  They stay in front of the stores behind them ("memory"): a row may be written where it was read.
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(static_cast<const char*>(p) + 16)
               : "memory");
}
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[4]) {
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[1]) {
  asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p) : "memory");
}
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[2]) {
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p) : "memory");
}
template <typename T, int VEC>
__device__ __forceinline__ Piece<T, VEC> load_piece(const T* p) {
  Piece<T, VEC> r;
  if constexpr (VEC == 1 && sizeof(T) == 2) r.w[0] = *reinterpret_cast<const uint16_t*>(p);
  else if constexpr (VEC == 1) r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  else load_words(p, r.w);
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, VEC>& r) {
  if constexpr (VEC == 1 && sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(r.w[0]);
  else if constexpr (VEC == 1) *reinterpret_cast<uint32_t*>(p) = r.w[0];
  else if constexpr (Piece<T, VEC>::WORDS == 1) *reinterpret_cast<uint32_t*>(p) = r.w[0];
  else if constexpr (Piece<T, VEC>::WORDS == 2) *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
  else {
#pragma unroll
    for (int i = 0; i < Piece<T, VEC>::WORDS; i += 4)
      reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(r.w[i], r.w[i + 1], r.w[i + 2], r.w[i + 3]);
  }
}
// fp32 values of a piece (bf16 widens by a shift)
template <typename T, int VEC>
__device__ __forceinline__ void widen(const Piece<T, VEC>& r, float (&f)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(r.w[i]);
    else f[i] = __uint_as_float(i % 2 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
  }
}
// rounds to nearest even where T is bf16: the only rounding of what leaves a kernel
template <typename T, int VEC>
__device__ __forceinline__ Piece<T, VEC> narrow(const float (&f)[VEC]) {
  Piece<T, VEC> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.w[i] = __float_as_uint(f[i]);
  } else if constexpr (VEC == 1) {
    r.w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[i], f[i + 1]);
      r.w[i / 2] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  return r;
}

// ---- host side of the entry points -----------------------------------------------------------

// What a context lends to the entry points outside api.cu.
int ctx_device(const emoe_ctx* ctx);
bool ctx_dependent_launch(const emoe_ctx* ctx);
int ctx_cuda_fail(emoe_ctx* ctx, cudaError_t e);
int* ctx_check_word(emoe_ctx* ctx);
char* ctx_workspace(emoe_ctx* ctx, size_t* bytes);

// The context's device is current, and launches may overlap with the kernel in front, while one of these lives.
class CallScope {
 public:
  explicit CallScope(emoe_ctx* ctx) {
    err_ = cudaGetDevice(&before_);
    if (err_ == cudaSuccess && before_ != ctx_device(ctx)) {
      err_ = cudaSetDevice(ctx_device(ctx));
      changed_ = err_ == cudaSuccess;
    }
    g_pdl_enabled = ctx_dependent_launch(ctx);
  }
  ~CallScope() {
    g_pdl_enabled = false;
    if (changed_) cudaSetDevice(before_);
  }
  CallScope(const CallScope&) = delete;
  CallScope& operator=(const CallScope&) = delete;
  cudaError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool changed_ = false;
  cudaError_t err_;
};

inline bool dtype_ok(int dtype) { return dtype == EMOE_DTYPE_F32 || dtype == EMOE_DTYPE_BF16; }
inline size_t dtype_size(int dtype) { return dtype == EMOE_DTYPE_F32 ? 4 : 2; }
inline bool ptr_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Stable counting sort of n ids by one cluster of CTAs (dispatch.cu): the outputs of emoe_permute.  counts and slot_of_pair may be null.
// rest: ids outside [0, E - 1) are sorted into the last of the E lists, and only those other than -1 set the check word; else ids
// outside [0, E) are dropped and set it.  write_perm: else only the places without a pair are written.
cudaError_t launch_sort_pairs(const int32_t* ids, int n, int E, bool rest, int32_t* counts, int32_t* off, int32_t* perm, bool write_perm, int32_t* slot_of_pair,
                              int* check_word, cudaStream_t st);

}  // namespace emoe

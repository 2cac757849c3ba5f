// What the calls around the decode step share: launch descriptors, the batch of sequences on the
// device, and the launchers the C ABI calls after it has validated every argument.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "prr.h"
#include "prr_batch.h"
#include "prr_device.h"

namespace prr {

struct CacheArgs {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int num_kv_heads, max_pages, page_size, page_shift;
};

struct RopeLaunch {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* positions;
  const double* freqs;
  void* q_out;
  CacheArgs c;
  BatchArgs b;
  int num_q_heads, rot_dim;
  float scale;
  int splits;  // waves per token (set by the launcher)
  bool bf16, e4m3, interleaved;
};

struct CacheReadLaunch {
  CacheArgs c;  // the codes
  const int32_t* page_table;
  void* k_out;
  void* v_out;
  int num_tokens, page_begin, pages;
  bool bf16;
};

struct PromptLaunch {
  const void* q;
  const void* k;
  const void* v;
  void* out_o;
  float* out_m;
  float* out_l;
  float* part_o;  // [nsplit][total_q * Hq][128] normalised, nsplit > 1
  float* part_ml;  // [nsplit][total_q * Hq][2] maximum (unscaled logits) and sum
  BatchArgs b;
  int num_kv_heads, group, max_pages, page_shift;
  int tiles;      // row tiles of one KV head (numbers: some sequences have fewer)
  int seq_tiles;  // row tiles of every sequence, or 0: numbered by their rows
  int nsplit, part_tiles;  // parts of a row tile's keys, of so many tiles of 64 tokens
  int waves;   // of a workgroup, 32 rows each
  uint32_t magic;  // divides by the group size
  bool bf16;
};

struct DecodeLaunch {
  const void* q;
  CacheArgs c;
  const int32_t* pages;
  const int32_t* page_count;
  float* out_o32;
  void* out_o;
  float* out_m;
  float* out_l;
  float* part_o;   // [n_seqs][Hkv][nsplit][G][128] normalised, nsplit > 1
  float* part_ml;  // [n_seqs][Hkv][nsplit][G][2] maximum (unscaled logits) and sum
  BatchArgs b;
  int group, cap;
  int nsplit, tiles_per_split;  // tiles of 16 tokens
  bool bf16, e4m3;
};

hipError_t launch_rope_append(RopeLaunch a, hipStream_t stream);
hipError_t launch_cache_read(const CacheReadLaunch& a, hipStream_t stream);
// how the work of a call is split (host rules, by sizes alone): sets tiles / nsplit / tiles_per_split
void plan_prompt(PromptLaunch& a);
void plan_decode(DecodeLaunch& a);
hipError_t launch_prompt(const PromptLaunch& a, hipStream_t stream);
hipError_t launch_decode(const DecodeLaunch& a, hipStream_t stream);

#ifdef __HIPCC__

// Launch of `f` with one argument struct; the error is the launch's own.
template <class A>
hipError_t launch_one(const void* f, dim3 grid, int threads, hipStream_t stream, const A& a) {
  void* args[] = {const_cast<A*>(&a)};
  return hipLaunchKernel(f, grid, dim3(threads), args, 0, stream);
}

// 1/sqrt(128), and with the change to powers of two
constexpr float kSoftmaxScale = 0.08838834764831845f;
constexpr float kSoftmaxScale2 = 0.08838834764831845f * kLog2e;

// 2^x to one unit in the last place; results below the smallest normal number are 0
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Storage of an infinity or a NaN.
template <bool BF16>
__device__ __forceinline__ bool non_finite(uint32_t bits16) {
  constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
  return (bits16 & kExp) == kExp;
}

// Two floats rounded to nearest even to the 16-bit type, packed.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (BF16) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(x), static_cast<__bf16>(y)});
  } else {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
    return __builtin_bit_cast(uint32_t, f16x2_t{static_cast<_Float16>(x), static_cast<_Float16>(y)});
  }
}

// Two e4m3 codes (the lower or upper half of a word) times a power of two, in the 16-bit type.
template <bool BF16, bool UPPER>
__device__ __forceinline__ uint32_t unpack_codes(uint32_t word, float scale) {
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, UPPER));
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, UPPER));
}

#endif

}  // namespace prr

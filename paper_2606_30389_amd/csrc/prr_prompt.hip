// Causal attention of packed prompts over the paged cache.
#include "prr_context.h"

namespace prr {

namespace {

// Rows are (token, query head of the KV head) pairs, token by token, so that the G heads that share
// keys and values share the loads too and a diagonal tile wastes little: a workgroup of NW waves takes
// 32 NW rows of one sequence and KV head, a wave 32 of them, and walks over the keys in tiles of 64
// tokens with the running maximum and sum of a softmax.
//
// S^T (64 tokens x 32 rows) = K Q^T in 32x32x16 products: lane 32h+n has row n's logits of tokens
// 8(i/4) + 4h + i%4 of each 32, i < 16, so a row's maximum is in two lanes.  O^T (128 channels x 32
// rows) = V^T P^T: the lane's own eight weights of 16 tokens are the right operand as they are, and
// V^T's tokens are read in that order, 4 tokens of one channel at a time, by transposing LDS loads.
// So no weight moves between lanes, and the rescale of a row is local to a lane.
//
// K and V tiles lie in LDS row by row (256 bytes), their 16-byte chunks permuted by the row: a read
// of one chunk of eight consecutive rows (K), or of 32 bytes of four rows (V), touches every bank once.
// Two buffers: a tile's successor is loaded into registers before its products and stored after
// them, one barrier per tile.
constexpr int kTokens = 64;
constexpr float kNoRef = -3e38f;
// a row's reference exponent is moved only when its maximum outgrows it by this much (powers of two):
// weights stay below 2^8, in range of either type, and the accumulators are rarely rescaled
constexpr float kSlack = 8.0f;

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

template <bool BF16>
__device__ __forceinline__ f32x16_t mfma32(const u32x4_t& a, const u32x4_t& b, f32x16_t c) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0,
                                                  0, 0);
  }
}

typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ float max_halves(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The sequence and the row tile in it of tile number `tile` of the batch; false: no such tile.
__device__ __forceinline__ bool find_tile(const PromptLaunch& a, int rows, int tile, int& s, int& local, Seq& sq) {
  const auto tiles_of = [&](const Seq& x) { return ((x.q1 - x.q0) * a.group + rows - 1) / rows; };
  if (a.b.n_seqs == 1) {
    s = 0;
    sq = seq_at(a.b, 0);
    const int n = tiles_of(sq);
    local = n - 1 - tile;
    return tile < n;
  }
  int base = 0;
  for (int s0 = 0; s0 < a.b.n_seqs; s0 += kWave) {
    const int x = s0 + lane_id();
    const int n = x < a.b.n_seqs ? tiles_of(seq_at(a.b, x)) : 0;
    const int inc = wave_inclusive_scan(n);
    const uint64_t past = __ballot(base + inc > tile);
    if (past) {
      const int at = __builtin_ctzll(past);
      s = s0 + at;
      sq = seq_at(a.b, s);
      // the last rows of a sequence have the most keys: they are taken first
      local = base + __builtin_amdgcn_readlane(inc, at) - 1 - tile;
      return true;
    }
    base += __builtin_amdgcn_readlane(inc, kWave - 1);
  }
  return false;
}

template <bool BF16, int NW>
__global__ __launch_bounds__(NW * kWave) void prompt_kernel(const PromptLaunch a) {
  constexpr int kRows = 32 * NW;
  constexpr int kPass = 16 / NW;  // 16-byte chunks of a K (or V) tile per thread
  __shared__ __align__(16) uint16_t lds[2][2][kTokens * kHeadDim];  // [buffer][K, V]
  const int t = threadIdx.x, lane = lane_id(), w = __builtin_amdgcn_readfirstlane(t / kWave);
  const int n = lane & 31, hf = lane >> 5;
  const float kNegInf = -__builtin_inff();
  const int G = a.group;

  const int h = blockIdx.x % a.num_kv_heads, part = blockIdx.y;
  int s, local;
  Seq sq;
  if (!find_tile(a, kRows, blockIdx.x / a.num_kv_heads, s, local, sq)) return;
  const int rows = (sq.q1 - sq.q0) * G;
  const int row0 = local * kRows;
  const int first = sq.kv - (sq.q1 - sq.q0);  // position of the sequence's first new token
  // this lane's row, the positions of the wave's rows, and the keys that the workgroup needs
  const int row = min(row0 + 32 * w + n, rows - 1);
  const bool live = row0 + 32 * w + n < rows;
  const int tok = row / G, head = row - tok * G;
  const int pos = first + tok;
  const int wave_lo = first + min(row0 + 32 * w, rows - 1) / G;
  const int wave_hi = row0 + 32 * w < rows ? first + min(row0 + 32 * w + 31, rows - 1) / G : -1;
  const int keys = max(0, first + min(row0 + kRows - 1, rows - 1) / G + 1);
  const int ntiles = (keys + kTokens - 1) / kTokens;
  const int per = (ntiles + a.nsplit - 1) / a.nsplit;
  const int t0 = min(part * per, ntiles), t1 = min(t0 + per, ntiles);

  const int64_t out_row = ((int64_t)(sq.q0 + tok) * a.num_kv_heads + h) * G + head;
  u32x4_t qf[8];
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + out_row * kHeadDim + 8 * hf;
#pragma unroll
  for (int x = 0; x < 8; ++x) qf[x] = *reinterpret_cast<const u32x4_t*>(q + 16 * x);

  f32x16_t acc[4];
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[cb][i] = 0.0f;
  float mx = kNegInf, ref = kNoRef, l = 0.0f;

  // loads: thread t takes chunk t%16 of rows t/16 + 4 NW x
  const int chunk = t & 15, lrow = t >> 4;
  const int psz = 1 << a.page_shift;
  const int64_t head_row = (int64_t)h * a.max_pages << a.page_shift;
  const auto cache_row = [&](int tile, int x) {
    const int p = min(tile * kTokens + lrow + 4 * NW * x, keys - 1);
    const int phys = phys_page(a.b.page_table, a.b.table_stride, a.max_pages, s, p >> a.page_shift);
    return (head_row + ((int64_t)max(phys, 0) << a.page_shift) + (p & (psz - 1))) * kHeadDim + chunk * 8;
  };
  u32x4_t kr[kPass], vr[kPass];
  int64_t at[kPass];
  const auto load = [&]() {
#pragma unroll
    for (int x = 0; x < kPass; ++x) {
      kr[x] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.k) + at[x]);
      vr[x] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.v) + at[x]);
    }
  };
  const auto store = [&](int buf) {
#pragma unroll
    for (int x = 0; x < kPass; ++x) {
      const int r = lrow + 4 * NW * x;
      *reinterpret_cast<u32x4_t*>(&lds[buf][0][r * kHeadDim + ((chunk ^ (r & 15)) * 8)]) = kr[x];
      *reinterpret_cast<u32x4_t*>(&lds[buf][1][r * kHeadDim + ((chunk ^ ((r & 7) << 1)) * 8)]) = vr[x];
    }
  };

  // LDS offsets (elements) of this lane's operands; k-steps and channel blocks flip chunk bits
  const int koff = n * kHeadDim + ((hf ^ (n & 15)) * 8);
  const int vi = lane & 15, vg = (lane >> 4) & 1;
  const int vrow = 4 * hf + (vi >> 2);
  const int voff = vrow * kHeadDim + (((2 * vg + ((vi >> 1) & 1)) ^ ((vrow & 7) << 1)) * 8) + (vi & 1) * 4;

  if (t0 < t1) {
#pragma unroll
    for (int x = 0; x < kPass; ++x) at[x] = cache_row(t0, x);
    load();
    store(0);
  }
  __syncthreads();
  for (int tile = t0; tile < t1; ++tile) {
    const int buf = (tile - t0) & 1;
    if (tile + 1 < t1) {
#pragma unroll
      for (int x = 0; x < kPass; ++x) at[x] = cache_row(tile + 1, x);
      load();
    }
    const int base = tile * kTokens;
    if (base <= wave_hi) {
      f32x16_t sc[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const u32x4_t kf = *reinterpret_cast<const u32x4_t*>(&lds[buf][0][(koff ^ (x * 16)) + b * 32 * kHeadDim]);
          sc[b] = mfma32<BF16>(kf, qf[x], sc[b]);
        }
      }
      if (base + kTokens - 1 > wave_lo) {  // some of the tokens come after some of the rows
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            sc[b][i] = base + 32 * b + 8 * (i / 4) + 4 * hf + i % 4 > pos ? kNegInf : sc[b][i];
      }
      float top = sc[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
      mx = fmaxf(mx, max_halves(top));
      if (__any(mx * kSoftmaxScale2 > ref + kSlack)) {
        const float next = mx == kNegInf ? ref : mx * kSoftmaxScale2;
        const float alpha = exp2_hw(ref - next);
        l *= alpha;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) acc[cb] *= alpha;
        ref = next;
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[b][i] = exp2_hw(fmaf(sc[b][i], kSoftmaxScale2, -ref));
          l += sc[b][i];
        }
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // 16 tokens
        const int b = x >> 1, i = 8 * (x & 1);
        const u32x4_t pf = {pack2<BF16>(sc[b][i], sc[b][i + 1]), pack2<BF16>(sc[b][i + 2], sc[b][i + 3]),
                            pack2<BF16>(sc[b][i + 4], sc[b][i + 5]), pack2<BF16>(sc[b][i + 6], sc[b][i + 7])};
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          uint16_t* v = &lds[buf][1][(voff ^ (cb * 32)) + x * 16 * kHeadDim];
          const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v);
          const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(v + 8 * kHeadDim));
          const uint2 a0 = __builtin_bit_cast(uint2, lo), a1 = __builtin_bit_cast(uint2, hi);
          acc[cb] = mfma32<BF16>(u32x4_t{a0.x, a0.y, a1.x, a1.y}, pf, acc[cb]);
        }
      }
    }
    if (tile + 1 < t1) store(buf ^ 1);
    __syncthreads();
  }

  l = sum_halves(l);
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  // l relative to the logit itself, not to its rounded product with the scale (and the slack)
  const float exact = mx == kNegInf ? 0.0f : l * exp2_hw(-fmaf(mx, kSoftmaxScale2, -ref));
  if (!live) return;
  if (a.nsplit == 1) {
    uint16_t* o = static_cast<uint16_t*>(a.out_o) + out_row * kHeadDim + 4 * hf;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<uint2*>(o + 32 * cb + 2 * i) =
            make_uint2(pack2<BF16>(acc[cb][i] * inv, acc[cb][i + 1] * inv),
                       pack2<BF16>(acc[cb][i + 2] * inv, acc[cb][i + 3] * inv));
    if (a.out_m && hf == 0) {
      a.out_m[out_row] = mx * kSoftmaxScale;
      a.out_l[out_row] = exact;
    }
  } else {
    const int64_t x = (int64_t)part * a.b.total_q * a.num_kv_heads * G + out_row;
    float* o = a.part_o + x * kHeadDim + 4 * hf;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(o + 32 * cb + 2 * i) =
            make_float4(acc[cb][i] * inv, acc[cb][i + 1] * inv, acc[cb][i + 2] * inv, acc[cb][i + 3] * inv);
    if (hf == 0) {
      a.part_ml[2 * x] = mx;
      a.part_ml[2 * x + 1] = exact;
    }
  }
}

// The parts of a row: 32 threads a row, four channels each.
template <bool BF16>
__global__ __launch_bounds__(256) void merge_prompt_kernel(const PromptLaunch a) {
  const int64_t rows = (int64_t)a.b.total_q * a.num_kv_heads * a.group;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int c4 = (threadIdx.x & 31) * 4;
  const float kNegInf = -__builtin_inff();
  const int end = a.b.cu_q ? min(a.b.cu_q[a.b.n_seqs], a.b.total_q) : a.b.n_seqs;
  if (row >= (int64_t)end * a.num_kv_heads * a.group) return;
  float mx = kNegInf;
  for (int p = 0; p < a.nsplit; ++p) mx = fmaxf(mx, a.part_ml[2 * (p * rows + row)]);
  float sum = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < a.nsplit; ++p) {
    const int64_t at = p * rows + row;
    const float m = a.part_ml[2 * at], l = a.part_ml[2 * at + 1];
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + at * kHeadDim + c4);
    const float f = m == kNegInf ? 0.0f : l * exp2_hw((m - mx) * kSoftmaxScale2);
    if (f != 0.0f) {
      sum += f;
      o.x += f * y.x;
      o.y += f * y.y;
      o.z += f * y.z;
      o.w += f * y.w;
    }
  }
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out_o) + row * kHeadDim + c4) =
      make_uint2(pack2<BF16>(o.x * inv, o.y * inv), pack2<BF16>(o.z * inv, o.w * inv));
  if (a.out_m && c4 == 0) {
    a.out_m[row] = mx * kSoftmaxScale;
    a.out_l[row] = sum;
  }
}

constexpr int kWaves = 8;

}  // namespace

void plan_prompt(PromptLaunch& a) {
  const int rows = 32 * kWaves;
  const int64_t packed = (int64_t)a.b.total_q * a.group / rows + a.b.n_seqs;
  const int64_t each = (int64_t)a.b.n_seqs * (((int64_t)a.b.max_q * a.group + rows - 1) / rows);
  a.tiles = (int)min(packed, each);
  // fewer workgroups than CUs: the keys are cut into parts of at least eight tiles
  const int64_t units = (int64_t)a.tiles * a.num_kv_heads;
  const int64_t key_tiles = ((int64_t)a.b.max_kv + kTokens - 1) / kTokens;
  a.nsplit = (int)max((int64_t)1, min((int64_t)256 / max(units, (int64_t)1), key_tiles / 8));
}

hipError_t launch_prompt(const PromptLaunch& a, hipStream_t stream) {
  const void* f = a.bf16 ? (const void*)prompt_kernel<true, kWaves> : (const void*)prompt_kernel<false, kWaves>;
  const hipError_t e = launch_one(f, dim3(a.tiles * a.num_kv_heads, a.nsplit), kWaves * kWave, stream, a);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t rows = (int64_t)a.b.total_q * a.num_kv_heads * a.group;
  return launch_one(a.bf16 ? (const void*)merge_prompt_kernel<true> : (const void*)merge_prompt_kernel<false>,
                    dim3((unsigned)((rows + 7) / 8)), 256, stream, a);
}

}  // namespace prr

// Attention of packed prompts over the paged cache: causal, or with capped, biased and masked scores.
#pragma once

#include <type_traits>

#include "prr_context.h"
#include "prr_shape.h"

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
// The weights are rounded to the 16-bit type, once, as the output is: the largest error of 509 tokens over 65536 is
// 1.4 times that of float32 weights.  A second term would make 48 products of a tile's 32.
//
// K and V tiles lie in LDS row by row, the rows padded by 16 (K) and 64 bytes (V), so that a read of 16
// bytes of eight rows, or of 32 bytes of four, touches every bank once at an immediate offset
// (permuted chunks instead: 28% of the LDS cycles were conflicts).  Two buffers each; global loads run
// a tile ahead in registers.
//
// A tile is a matrix phase (the tile before with V, this tile with K: 32 products, 1024 cycles) and a
// vector phase (its softmax, about as long).  A SIMD has two waves of the workgroup, w and w + 4; the
// second half of the waves runs one phase behind the first, barriers between the phases, so that one
// wave's products run under the other's softmax.  16384 tokens, 32 / 2 heads, bf16: 2154 us with all
// waves in step (MFMA 46% of the cycles, VALU 45%, one after the other), 1945 in turns: 1.13 PFLOP/s,
// where a 16384^3 library product reaches 1.38.  The clock falls from 2.15 to 1.8 GHz meanwhile: power
// bounds it, and schedules with fewer stalls but more instructions (four sums and maxima side by side,
// operands read further ahead) come out 1-3% slower.
//
// Up to 1024 tokens, four waves a workgroup, two workgroups a CU, which start and end (about 9 us a
// workgroup) under each other's work instead of taking turns: 32 sequences of 512 tokens, 32 / 8 heads, 140 us
// (eight waves: 152), 1024 tokens 29 (39); 2048 tokens 61 (58), 16384 tokens 2118 (1916).  (plan_prompt: with a shape.)
//
// SHAPE (prr_shape.h): a row sees an interval of keys, [lo, hi).  The workgroup's tiles are those that its rows'
// intervals touch; a tile that every row of a wave sees whole takes the path without comparisons.  Caps and slopes
// are applied to the logits in the units of q.k, so that everything behind them is the same.
constexpr int kTokens = 64;
constexpr int kKPitch = kHeadDim + 8, kVPitch = kHeadDim + 32;  // elements
constexpr float kNoRef = -3e38f;
// A row's weights are relative to a reference exponent that puts its maximum at 2^kTop and is moved only when
// the maximum outgrows that by 2^kSlack, so that the accumulators are rarely rescaled.  float16 weights lie at
// the top of their range (below 2^15): their step of 2^-24 is 2^-35 of the row's maximum or less (with the
// maximum at 1, keys 17 nats below it were counted in the sum but not in the output).
template <bool BF16>
constexpr float kTop = BF16 ? 0.0f : 11.0f;
template <bool BF16>
constexpr float kSlack = BF16 ? 8.0f : 4.0f;

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

// x / G for 0 <= x < 2^28 (G <= 16): magic = ceil(2^32 / G), off by less than G / 2^32 of x; 0 stands for G = 1
__device__ __forceinline__ int over_group(int x, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)x, magic) : x; }

// The sequence and the row tile in it of the batch's tile number `tile`; false: none.  Tiles are numbered by a
// rule that needs no sums over the sequences.  With seq_tiles, every sequence has so many, and the last tile
// of all sequences comes first, as it has the most keys.  Without, sequence s has the numbers from
// floor(cu[s] G / rows) + s on: the next sequence's begin at least ceil(q_len G / rows) later.
__device__ __forceinline__ bool find_tile(const PromptLaunch& a, int rows_log2, int tile, int& s, int& local, Seq& sq) {
  s = 0;
  local = tile;
  if (a.b.n_seqs > 1 && a.seq_tiles) {
    local = tile / a.b.n_seqs;
    s = tile - local * a.b.n_seqs;
  } else if (a.b.n_seqs > 1) {
    const auto begin_of = [&](int x) { return (int)(((int64_t)a.b.cu_q[x] * a.group) >> rows_log2) + x; };
    for (int n = a.b.n_seqs; n > 1;) {  // 64 candidates at a time
      const int step = (n + kWave - 1) / kWave, lane = lane_id();
      const bool ok = lane * step < n && begin_of(s + lane * step) <= tile;
      const int at = max(__popcll(__ballot(ok)) - 1, 0) * step;
      s += at;
      n = min(step, n - at);
    }
    local -= begin_of(s);
  }
  sq = seq_at(a.b, s);
  const int n = ((sq.q1 - sq.q0) * a.group + (1 << rows_log2) - 1) >> rows_log2;
  local = (a.seq_tiles ? a.seq_tiles : n) - 1 - local;
  return local >= 0 && local < n;
}

template <bool BF16, bool PAGED, int NW, bool TURNS, int SHAPE = 0>
__global__ __launch_bounds__(NW * kWave, 2) void prompt_kernel(const PromptLaunch a) {
  constexpr int kRows = 32 * NW;
  constexpr int kPass = 16 / NW;  // 16-byte chunks of a K (or V) tile per thread
  __shared__ __align__(16) uint16_t lds[2][kTokens * (kKPitch + kVPitch)];  // [buffer] K, V
  __shared__ int any_bad;  // non-finite values were set aside
  __shared__ int ranges[SHAPE ? 4 : 1][NW];
  const int t = threadIdx.x, lane = lane_id(), w = __builtin_amdgcn_readfirstlane(t / kWave);
  const int n = lane & 31, hf = lane >> 5;
  const float kNegInf = -__builtin_inff();
  const int G = a.group;

  const int h = blockIdx.x % a.num_kv_heads, part = blockIdx.y;
  int s, local;
  Seq sq;
  if (!find_tile(a, NW == 8 ? 8 : 7, blockIdx.x / a.num_kv_heads, s, local, sq)) return;
  const int rows = (sq.q1 - sq.q0) * G;
  const int row0 = local * kRows;
  const int first = sq.kv - (sq.q1 - sq.q0);  // position of the sequence's first new token
  // this lane's row, the positions of the wave's rows, and the keys that the workgroup needs
  const int row = min(row0 + 32 * w + n, rows - 1);
  const bool live = row0 + 32 * w + n < rows;
  const int tok = over_group(row, a.magic), head = row - tok * G;
  const int pos = first + tok;
  int keys, ntiles, t0, t1;
  int whole0 = 0, whole1;  // tiles [whole0, whole1): whose tokens every row of the wave sees
  int all0 = 0, all1;      // the same for every row of the workgroup
  [[maybe_unused]] Span sp;
  [[maybe_unused]] float slope = 0.0f;
  if constexpr (SHAPE) {
    sp = span_of(a.sh, pos, sq.q0 + tok, s, sq.kv);
    const bool sees = sp.lo < sp.hi;
    const uint32_t r0 = wave_umin(sees ? sp.lo : 0x7fffffffu), r1 = wave_umax(sees ? sp.hi : 0), r2 = wave_umax(sp.lo),
                   r3 = wave_umin(sp.hi);
    whole0 = (int)(r2 + kTokens - 1) / kTokens;
    whole1 = (int)r3 / kTokens;
    if (lane == 0) {
      ranges[0][w] = (int)r0;
      ranges[1][w] = (int)r1;
      ranges[2][w] = (int)r2;
      ranges[3][w] = (int)r3;
    }
    if (t == 0) any_bad = 0;
    __syncthreads();
    int lo = 0x7fffffff, lo_last = 0, hi_first = 0x7fffffff;
    keys = 0;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      lo = min(lo, ranges[0][x]);
      keys = max(keys, ranges[1][x]);
      lo_last = max(lo_last, ranges[2][x]);
      hi_first = min(hi_first, ranges[3][x]);
    }
    all0 = (lo_last + kTokens - 1) / kTokens;
    all1 = hi_first / kTokens;
    ntiles = (keys + kTokens - 1) / kTokens;
    t0 = min(min(lo, keys) / kTokens + part * a.part_tiles, ntiles);
    if constexpr (SHAPE & kShapeSlopes) slope = slope_of<SHAPE>(a.sh, h * G + head);
  } else {
    const int wave_lo = first + over_group(min(row0 + 32 * w, rows - 1), a.magic);
    keys = max(0, first + over_group(min(row0 + kRows - 1, rows - 1), a.magic) + 1);
    ntiles = (keys + kTokens - 1) / kTokens;
    t0 = min(part * a.part_tiles, ntiles);
    whole1 = (wave_lo + 1) / kTokens;
    all1 = (first + over_group(row0, a.magic) + 1) / kTokens;
    if (t == 0) any_bad = 0;
    if (TURNS) __syncthreads();  // (else the first barrier below comes before the first values)
  }
  t1 = min(t0 + a.part_tiles, ntiles);

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

  // loads: thread t takes chunk t%16 of rows t/16 + 4 NW x; the four rows of a wave lie in one page
  const int chunk = t & 15, lrow = t >> 4;
  const int pmask = (1 << a.page_shift) - 1;
  const int64_t head_byte = ((int64_t)h * a.max_pages << a.page_shift) * (2 * kHeadDim);
  const char* const kbase = static_cast<const char*>(a.k) + head_byte;
  const char* const vbase = static_cast<const char*>(a.v) + head_byte;
  // The physical pages of the wave's rows of a tile, those of pass x in lane x: looked up a tile before
  // they are used, so that nothing waits for them.
  const auto lookup = [&](int tile) {
    const int p = min(tile * kTokens + 4 * w + 4 * NW * (lane % kPass), keys - 1) >> a.page_shift;
    if constexpr (PAGED) return a.b.page_table[(int64_t)s * a.b.table_stride + p];
    return p;
  };
  const auto pages_of = [&](int found, int64_t (&page)[kPass]) {
#pragma unroll
    for (int x = 0; x < kPass; ++x) {
      const int p = __builtin_amdgcn_readlane(found, x);
      page[x] = (int64_t)((uint32_t)p < (uint32_t)a.max_pages ? p : 0) << (a.page_shift + 8);
    }
  };
  u32x4_t kr[kPass], vr[kPass];
  const auto load = [&](u32x4_t (&r)[kPass], const char* base, int tile, const int64_t (&page)[kPass]) {
#pragma unroll
    for (int x = 0; x < kPass; ++x) {
      const uint32_t off = (uint32_t)(min(tile * kTokens + lrow + 4 * NW * x, keys - 1) & pmask) * 256 + chunk * 16;
      r[x] = *reinterpret_cast<const u32x4_t*>(base + page[x] + off);
    }
  };
  int64_t pg0[kPass], pg1[kPass];  // pages of the next tiles
  const auto store_k = [&](int buf) {
#pragma unroll
    for (int x = 0; x < kPass; ++x) *reinterpret_cast<u32x4_t*>(&lds[buf][(lrow + 4 * NW * x) * kKPitch + chunk * 8]) = kr[x];
  };
  // In tiles that some row sees in part, a non-finite value would reach the rows that do not see it as 0 * v:
  // it is stored as 0 and added to the rows that see it at the end.
  const auto store_v = [&](int buf, int tile) {
    if ((SHAPE && tile < all0) || tile >= all1) {
      // (an exponent of all ones carries into its half's sign bit)
      constexpr uint32_t kExp = BF16 ? 0x7f807f80u : 0x7c007c00u, kOne = BF16 ? 0x00800080u : 0x04000400u;
      uint32_t carry = 0;
#pragma unroll
      for (int x = 0; x < kPass; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) carry |= (vr[x][i] & kExp) + kOne;
      if (carry & 0x80008000u) {
        any_bad = 1;
#pragma unroll
        for (int x = 0; x < kPass; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            vr[x][i] &= (non_finite<BF16>(vr[x][i]) ? 0u : 0xffffu) | (non_finite<BF16>(vr[x][i] >> 16) ? 0u : 0xffff0000u);
      }
    }
#pragma unroll
    for (int x = 0; x < kPass; ++x)
      *reinterpret_cast<u32x4_t*>(&lds[buf][kTokens * kKPitch + (lrow + 4 * NW * x) * kVPitch + chunk * 8]) = vr[x];
  };

  // LDS offsets (elements) of this lane's operands
  const int koff = n * kKPitch + hf * 8;
  const int vi = lane & 15, vg = (lane >> 4) & 1;
  const int voff = kTokens * kKPitch + (4 * hf + (vi >> 2)) * kVPitch + 16 * vg + 4 * (vi & 3);

  f32x16_t sc[2];   // logits of the current tile
  u32x4_t pf[4];    // weights of the tile before
#pragma unroll
  for (int x = 0; x < 4; ++x) pf[x] = u32x4_t{0, 0, 0, 0};

  const auto qk_step = [&](f32x16_t (&d)[2], int buf, int b, int x) {
    const u32x4_t kf = *reinterpret_cast<const u32x4_t*>(&lds[buf][koff + x * 16 + b * 32 * kKPitch]);
    d[b] = mfma32<BF16>(kf, qf[x], d[b]);
  };
  const auto pv_step = [&](int buf, int x, int cb) {
    uint16_t* v = &lds[buf][voff + cb * 32 + x * 16 * kVPitch];
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v);
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(v + 8 * kVPitch));
    const uint2 a0 = __builtin_bit_cast(uint2, lo), a1 = __builtin_bit_cast(uint2, hi);
    acc[cb] = mfma32<BF16>(u32x4_t{a0.x, a0.y, a1.x, a1.y}, pf[x], acc[cb]);
  };
  // Matrix phase: the tile before with V, this tile with K.
  const auto matrix = [&](int tile) {
    const int buf = (tile - t0) & 1;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
      for (int x = 0; x < 8; ++x) qk_step(sc, buf, b, x);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) pv_step(buf ^ 1, x, cb);
    asm volatile("" : "+v"(sc[0]), "+v"(sc[1]), "+v"(acc[0]), "+v"(acc[1]), "+v"(acc[2]), "+v"(acc[3]));
    __builtin_amdgcn_s_setprio(0);
  };
  // Vector phase: the softmax of this tile.
  const auto vector = [&](int tile, auto masked) {
    // Where nothing comes between the cap and the exponent, the cap's product is the exponent's; the cap does not change
    // the order of logits, so the largest is known before.
    constexpr bool kFold = (SHAPE & kShapeCap) && !(SHAPE & kShapeSlopes) && !masked.value;
    if constexpr ((SHAPE & kShapeCap) && !kFold) {
      float most = 0.0f;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(sc[b][i]));
      if ((SHAPE & kShapeSlopes) && a.sh.wide) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[b][i] = cap_wide(sc[b][i], a.sh);
      } else if (__all(most < a.sh.small)) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[b][i] = cap_small(sc[b][i], a.sh);
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[b][i] = cap_any(sc[b][i], a.sh);
      }
    }
    if constexpr (SHAPE & kShapeSlopes) {
      const float ahead = (float)(tile * kTokens + 4 * hf - pos);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = fmaf(-slope, fabsf(ahead + (float)(32 * b + 8 * (i / 4) + i % 4)), sc[b][i]);
    }
    if constexpr (masked.value && SHAPE) {
      const uint32_t base = (uint32_t)(tile * kTokens + 4 * hf - sp.lo), seen = (uint32_t)(sp.hi - sp.lo);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = base + (uint32_t)(32 * b + 8 * (i / 4) + i % 4) < seen ? sc[b][i] : kNegInf;
    } else if constexpr (masked.value) {
      const int base = tile * kTokens;
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
    [[maybe_unused]] bool near = false;
    if constexpr (kFold) {
      float least = sc[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) least = fminf(least, sc[b][i]);
      near = __all(fmaxf(fabsf(top), fabsf(least)) < a.sh.small);
      top = cap_any(top, a.sh);
    }
    mx = fmaxf(mx, max_halves(top));
    const float scaled = mx * kSoftmaxScale2;
    const bool grown = scaled > ref + (kTop<BF16> + kSlack<BF16>);
    if (__any(grown)) {
      const float next = grown ? scaled - kTop<BF16> : ref;
      const float alpha = exp2_hw(ref - next);
      ref = next;
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) acc[cb] *= alpha;
    }
    const auto weights = [&](auto&& exponent) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[b][i] = exp2_hw(exponent(sc[b][i]));
          l += sc[b][i];
        }
    };
    if constexpr (kFold) {
      if (near) {
        weights([&](float x) { return cap_exponent(x, ref, kSoftmaxScale2, true, a.sh); });
      } else {
        weights([&](float x) { return cap_exponent(x, ref, kSoftmaxScale2, false, a.sh); });
      }
    } else {
      weights([&](float x) { return fmaf(x, kSoftmaxScale2, -ref); });
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int b = x >> 1, i = 8 * (x & 1);
      pf[x] = u32x4_t{pack2<BF16>(sc[b][i], sc[b][i + 1]), pack2<BF16>(sc[b][i + 2], sc[b][i + 3]),
                      pack2<BF16>(sc[b][i + 4], sc[b][i + 5]), pack2<BF16>(sc[b][i + 6], sc[b][i + 7])};
      asm volatile("" : "+v"(pf[x]));
    }
  };
  const auto barrier = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    __builtin_amdgcn_sched_barrier(0);
  };

  if (t0 < t1) {
    const int late = TURNS && w >= NW / 2;  // this half of the waves runs a phase behind the other
    // what this wave stores in the vector phase of tile i: keys of tile i + 1 + late, values of i + late
    int found = lookup(t0);
    const int found1 = lookup(t0 + 1);
    pages_of(found, pg0);
    pages_of(found1, pg1);
    u32x4_t k0[kPass];
    load(k0, kbase, t0, pg0);
    load(kr, kbase, t0 + 1, pg1);
    load(vr, vbase, t0, pg0);
    found = lookup(t0 + 2);
#pragma unroll
    for (int x = 0; x < kPass; ++x)
      *reinterpret_cast<u32x4_t*>(&lds[0][(lrow + 4 * NW * x) * kKPitch + chunk * 8]) = k0[x];
    if (late) {
      store_k(1);
      store_v(0, t0);
#pragma unroll
      for (int x = 0; x < kPass; ++x) pg0[x] = pg1[x];
      pages_of(found, pg1);
      load(kr, kbase, t0 + 2, pg1);
      load(vr, vbase, t0 + 1, pg0);
      found = lookup(t0 + 3);
    }
    // (values of the tile before the first: the other buffer, all zero)
    {
      const u32x4_t z = {0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < kPass; ++x)
        *reinterpret_cast<u32x4_t*>(&lds[1][kTokens * kKPitch + (lrow + 4 * NW * x) * kVPitch + chunk * 8]) = z;
    }
    barrier();
    if (late) barrier();
    const int whole = min(t1, max(t0, whole1));
    const auto step = [&](int tile, auto masked) {
      matrix(tile);
      if (TURNS) barrier();
      const int kb = (tile - t0 + 1 + late) & 1;
      store_k(kb);
      store_v(kb ^ 1, tile + late);
#pragma unroll
      for (int x = 0; x < kPass; ++x) pg0[x] = pg1[x];
      pages_of(found, pg1);
      found = lookup(tile + 3 + late);
      load(kr, kbase, tile + 2 + late, pg1);
      load(vr, vbase, tile + 1 + late, pg0);
      vector(tile, masked);
      barrier();
    };
    int tile = t0;
    if constexpr (SHAPE)
      for (const int first_whole = min(whole, whole0); tile < first_whole; ++tile) step(tile, std::true_type{});
    for (; tile < whole; ++tile) step(tile, std::false_type{});
    for (; tile < t1; ++tile) step(tile, std::true_type{});
    if (TURNS && !late) barrier();
    const int buf = (t1 - 1 - t0) & 1;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) pv_step(buf, x, cb);
  }

  __syncthreads();
  if (any_bad) {  // what was set aside, to the rows that see it: whatever its weight, the result is not finite
    for (int p = (SHAPE ? t0 : max(all1, t0)) * kTokens; p < min(t1 * kTokens, keys); ++p) {
      if (SHAPE && p / kTokens >= all0 && p / kTokens < all1) continue;
      const int phys = phys_page(a.b.page_table, a.b.table_stride, a.max_pages, s, p >> a.page_shift);
      const char* v = vbase + ((int64_t)max(phys, 0) << (a.page_shift + 8)) + (int64_t)(p & pmask) * 256 + 8 * hf;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t x = *reinterpret_cast<const uint16_t*>(v + 64 * cb + 16 * (i / 4) + 2 * (i % 4));
          if (non_finite<BF16>(x) && (SHAPE ? p >= sp.lo && p < sp.hi : p <= pos)) acc[cb][i] += h2f<BF16>(x);
        }
    }
  }

  l = sum_halves(l);
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  // l relative to the logit itself, not to its rounded product with the scale (and the slack)
  const float exact = l == 0.0f || l != l ? l : l * exp2_hw(-fmaf(mx, kSoftmaxScale2, -ref));
  if (a.nsplit == 1) {
    // (the halves of a wave swap four of their eight channels, so that a store holds 16 bytes of a row)
    uint16_t* o = static_cast<uint16_t*>(a.out_o) + out_row * kHeadDim + 8 * hf;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 16; i += 8) {
        uint32_t r[4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const auto two = __builtin_amdgcn_permlane32_swap(
              pack2<BF16>(acc[cb][i + 2 * x] * inv, acc[cb][i + 2 * x + 1] * inv),
              pack2<BF16>(acc[cb][i + 4 + 2 * x] * inv, acc[cb][i + 5 + 2 * x] * inv), false, false);
          r[x] = two[0];
          r[2 + x] = two[1];
        }
        if (live) *reinterpret_cast<uint4*>(o + 32 * cb + 2 * i) = make_uint4(r[0], r[1], r[2], r[3]);
      }
    if (live && a.out_m && hf == 0) {
      a.out_m[out_row] = mx * kSoftmaxScale;
      a.out_l[out_row] = exact;
    }
  } else if (live) {
    const int64_t x = (int64_t)part * a.b.total_q * a.num_kv_heads * G + out_row;
    float* o = a.part_o + x * kHeadDim + 4 * hf;
    if (t0 < t1) {  // (the outputs of an empty part are not read)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(o + 32 * cb + 2 * i) =
              make_float4(acc[cb][i] * inv, acc[cb][i + 1] * inv, acc[cb][i + 2] * inv, acc[cb][i + 3] * inv);
    }
    if (hf == 0) {
      a.part_ml[2 * x] = l != l ? l : mx;  // (maxima pass over NaN: a state of NaN must not look empty)
      a.part_ml[2 * x + 1] = exact;
    }
  }
}

// The parts of a row: 32 threads hold its channels, four each; GROUPS such groups share the row's parts.
template <bool BF16, int GROUPS>
__global__ __launch_bounds__(256) void merge_prompt_kernel(const PromptLaunch a) {
  __shared__ __align__(16) float so[GROUPS][kHeadDim], sl[GROUPS];
  const int64_t rows = (int64_t)a.b.total_q * a.num_kv_heads * a.group;
  const int grp = GROUPS == 1 ? 0 : threadIdx.x >> 5;
  const int64_t row = GROUPS == 1 ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  const int c4 = (threadIdx.x & 31) * 4;
  const float kNegInf = -__builtin_inff();
  const int end = a.b.cu_q ? min(a.b.cu_q[a.b.n_seqs], a.b.total_q) : a.b.n_seqs;
  if (row >= (int64_t)end * a.num_kv_heads * a.group) return;
  float mx = kNegInf;
#pragma unroll 8
  for (int p = 0; p < a.nsplit; ++p) mx = fmaxf(mx, a.part_ml[2 * (p * rows + row)]);
  float sum = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p = grp; p < a.nsplit; p += GROUPS) {
    const int64_t at = p * rows + row;
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
    const float f = ml.x == kNegInf ? 0.0f : ml.y * exp2_hw((ml.x - mx) * kSoftmaxScale2);
    // (an empty part has no output: the first part's is read instead, which there always is)
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + (ml.x == kNegInf ? row : at) * kHeadDim + c4);
    sum += f;
    o.x += f != 0.0f ? f * y.x : 0.0f;
    o.y += f != 0.0f ? f * y.y : 0.0f;
    o.z += f != 0.0f ? f * y.z : 0.0f;
    o.w += f != 0.0f ? f * y.w : 0.0f;
  }
  if constexpr (GROUPS > 1) {
    *reinterpret_cast<float4*>(&so[grp][c4]) = o;
    if (c4 == 0) sl[grp] = sum;
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int x = 1; x < GROUPS; ++x) {
      const float4 y = *reinterpret_cast<const float4*>(&so[x][c4]);
      sum += sl[x];
      o.x += y.x;
      o.y += y.y;
      o.z += y.z;
      o.w += y.w;
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

template <bool BF16, int SHAPE>
const void* prompt_fn(bool paged, int waves) {
  if (paged)
    return waves == 8 ? (const void*)prompt_kernel<BF16, true, 8, true, SHAPE> : (const void*)prompt_kernel<BF16, true, 4, false, SHAPE>;
  return waves == 8 ? (const void*)prompt_kernel<BF16, false, 8, true, SHAPE> : (const void*)prompt_kernel<BF16, false, 4, false, SHAPE>;
}

}  // namespace

}  // namespace prr

// Attention of one token per sequence over its whole cache or over listed pages, with or without a shape of the scores.
#pragma once

#include "prr_context.h"
#include "prr_shape.h"

namespace prr {

namespace {

// The keys of a (sequence, KV head) are cut into tiles of 16 tokens, the tiles into runs of eight, and the
// runs are dealt out to the parts, one workgroup of eight waves each, so that all workgroups read one
// moving window of the cache (parts of consecutive tokens are 2% slower).  Wave w takes tile w of
// each run with an online softmax of its own, the next tile's loads issued before a tile is computed (more
// in flight is no faster: of the 20.0 us of a call over 2 x 131072 e4m3 tokens, 16 to 18 in this kernel and 2.3 to 4
// in the join, 18.6 remain when nothing is computed).  The wave
// states are merged in LDS; with more than one part, by merge_parts_kernel over the parts.
//
// Matrix products are those of the page-list attention (prr_sep.h, pv_tile): lane 16j+n has the logits of
// tokens 4j..4j+3 for query head n and channels 32j + 8i + cb of its output.  A key row's 16-byte
// pieces go to the four lanes of a load instruction in order, 64 bytes of a row at a time (64 bytes of a
// row to one lane, a load each 16: 8% slower).  32 sequences of up to 16K float16 tokens, 32 / 8 heads: 222 us, 5.4 TB/s.
//
// Weights: bfloat16 ones are three terms, all of float32's bits.  float16 ones are two, 22 bits, of numbers that
// a power of two per head and tile lifts to the top of float16's range: what is 2^-17 below the largest weight
// of its 16 tokens loses bits (2^-39 of it is the step), never what is below another tile's.  (Relative to
// the largest weight of all, 17 nats below it nothing was left of 131071 keys.)
//
// An e4m3 cache: codes are exact in either 16-bit type.  q.code is scaled by the key's power of two
// in float32.  The value's power of two 2^ev joins the weight, exactly: p 2^(ev - top + kHeadroom), top
// the largest ev so far.  A large scale says nothing about a row's other channels, so the weights of rows
// with far smaller scales have to keep their bits: the product runs in bfloat16, whose three-term weights
// have float32's bits and range, and weights up to 2^kHeadroom leave the lower 2^-126 to the others (2 x 131072
// tokens: 20.0 us, 19.5 with two float16 terms; 2 x 256 tiles 9.7, 9.4).
//
// SHAPE (prr_shape.h): the tiles are those from the first key on that the token sees, and rows before that key
// repeat it, so that nothing hidden is read or multiplied.
constexpr int NW = 8;  // waves of a workgroup
constexpr int kTile = 16;
constexpr float kNoRef = -3e38f;  // nothing seen yet: 2^(kNoRef - anything later) = 0
// (2^30 tokens of codes up to 448 stay below 2^(30 + 9 + 88) = 2^127)
constexpr int kHeadroom = 88;

template <bool E4M3>
struct TileData {
  u32x4_t k[E4M3 ? 2 : 4];
  u32x4_t v[4];  // E4M3: only .x, .y of each
  uint32_t ks, vs;
};

template <bool BF16>
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t& a, const u32x4_t& b, f32x4_t c) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0,
                                                  0, 0);
  }
}

// Tile `row0` (first cache row) with tokens [skip, valid) of its 16, one at least; the rows around them repeat the nearest.
template <bool E4M3>
__device__ __forceinline__ void load_tile(const CacheArgs& c, int64_t row0, int skip, int valid, TileData<E4M3>& d) {
  const int lane = lane_id(), j = lane >> 4, m = lane & 15;
  const auto near = [&](int x) { return max(min(x, valid - 1), skip); };
  if constexpr (E4M3) {
    const uint8_t* k = static_cast<const uint8_t*>(c.k) + (row0 + near(m)) * kHeadDim + 16 * j;
    d.k[0] = *reinterpret_cast<const u32x4_t*>(k);
    d.k[1] = *reinterpret_cast<const u32x4_t*>(k + 64);
    const uint8_t* v = static_cast<const uint8_t*>(c.v) + row0 * kHeadDim + 8 * m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>(v + near(4 * j + i) * kHeadDim);
      d.v[i][0] = w.x;
      d.v[i][1] = w.y;
    }
    d.ks = *reinterpret_cast<const uint32_t*>(c.k_scale + row0 + 4 * j);
    d.vs = *reinterpret_cast<const uint32_t*>(c.v_scale + row0 + 4 * j);
  } else {
    const uint16_t* k = static_cast<const uint16_t*>(c.k) + (row0 + near(m)) * kHeadDim + 8 * j;
#pragma unroll
    for (int s = 0; s < 4; ++s) d.k[s] = *reinterpret_cast<const u32x4_t*>(k + 32 * s);
    const uint16_t* v = static_cast<const uint16_t*>(c.v) + row0 * kHeadDim + 8 * m;
#pragma unroll
    for (int i = 0; i < 4; ++i) d.v[i] = *reinterpret_cast<const u32x4_t*>(v + near(4 * j + i) * kHeadDim);
  }
}

// A wave's running state: per lane the head n = lane % 16.  mx the largest logit (unscaled q.k), ref
// the exponent (powers of two) that l and acc are relative to, l this lane's part of the sum; E4M3: top
// the largest scale byte of the values, acc relative to 2^(top - 127 - kHeadroom) too.
struct WaveState {
  f32x4_t acc[8];
  float mx, ref, l;
  int top;
};

// back: how far the tile's first token lies behind the query's.
template <bool BF16, bool E4M3, int SHAPE>
__device__ __forceinline__ void attend_tile(const TileData<E4M3>& d, const u32x4_t (&qf)[4], int skip, int valid, int back,
                                            float slope, const ShapeArgs& sh, WaveState& st) {
  const int j = lane_id() >> 4;
  const float kNegInf = -__builtin_inff();
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    if constexpr (E4M3) {
      const uint32_t a = d.k[x >> 1][2 * (x & 1)], b = d.k[x >> 1][2 * (x & 1) + 1];
      const u32x4_t kf = {unpack_codes<BF16, false>(a, 1.0f), unpack_codes<BF16, true>(a, 1.0f),
                          unpack_codes<BF16, false>(b, 1.0f), unpack_codes<BF16, true>(b, 1.0f)};
      s = mfma16<BF16>(kf, qf[x], s);
    } else {
      s = mfma16<BF16>(d.k[x], qf[x], s);
    }
  }
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool live = 4 * j + i < valid && (!SHAPE || 4 * j + i >= skip);
    if constexpr (E4M3) s[i] *= __uint_as_float(((d.ks >> (8 * i)) & 0xffu) << 23);
    if constexpr (SHAPE & kShapeCap) s[i] = cap_exact(s[i], sh);
    if constexpr (SHAPE & kShapeSlopes) s[i] = fmaf(-slope, (float)(back - 4 * j - i), s[i]);
    s[i] = live ? s[i] : kNegInf;
    top = fmaxf(top, s[i]);
  }
  top = max_rows(top);
  st.mx = fmaxf(st.mx, top);
  const float ref = st.mx == kNegInf ? st.ref : st.mx * kSoftmaxScale2;
  const float alpha = exp2_hw(st.ref - ref);
  st.l *= alpha;
  if (__any(ref != st.ref)) {
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) st.acc[cb] *= alpha;
  }
  st.ref = ref;
  if constexpr (E4M3) {
    int vtop = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) vtop = max(vtop, 4 * j + i < valid && (!SHAPE || 4 * j + i >= skip) ? (int)((d.vs >> (8 * i)) & 0xffu) : 0);
    if (__any(vtop > st.top)) {
      const int next = max(st.top, (int)max_rows((float)vtop));
#pragma unroll
      for (int cb = 0; cb < 8; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.acc[cb][i] = ldexpf(st.acc[cb][i], st.top - next);
      st.top = next;
    }
  }
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float p = exp2_hw(fmaf(s[i], kSoftmaxScale2, -ref));
    st.l += p;
    w[i] = E4M3 ? ldexpf(p, (int)((d.vs >> (8 * i)) & 0xffu) - st.top + kHeadroom) : p;
  }
  if constexpr (E4M3) {
    u32x4_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = u32x4_t{unpack_codes<true, false>(d.v[i][0], 1.0f), unpack_codes<true, true>(d.v[i][0], 1.0f),
                     unpack_codes<true, false>(d.v[i][1], 1.0f), unpack_codes<true, true>(d.v[i][1], 1.0f)};
    pv_tile<true, 3>(st.acc, v, w);
  } else if constexpr (BF16) {
    pv_tile<true, 3>(st.acc, d.v, w);
  } else {
    // the largest of the tile's weights to 2^14..2^15, and the tile's sums back by as much
    const int by = 15 - __builtin_amdgcn_frexp_expf(exp2_hw(fmaf(top, kSoftmaxScale2, -ref)));
    f32x4_t sum[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = ldexpf(w[i], by);
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) sum[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    pv_tile<false>(sum, d.v, w);
    const float back = ldexpf(1.0f, -by);
#pragma unroll
    for (int cb = 0; cb < 8; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[cb][i] = fmaf(sum[cb][i], back, st.acc[cb][i]);
  }
}

// The first key that the token of sequence s sees (kv: none).
template <int SHAPE>
__device__ __forceinline__ int first_key(const DecodeLaunch& a, int s, int kv) {
  if constexpr (SHAPE) return kv > 0 ? span_of(a.sh, kv - 1, s, s, kv).lo : 0;
  return 0;
}
// Tiles of (sequence s, KV head h); without lists, from that of the first key on.
__device__ __forceinline__ int key_tiles(const DecodeLaunch& a, int s, int h, int lo, int kv) {
  if (!a.pages) return lo < kv ? (kv + kTile - 1) / kTile - lo / kTile : 0;
  return min(max(a.page_count[(size_t)s * a.c.num_kv_heads + h], 0), a.cap) << (a.c.page_shift - 4);
}
__device__ __forceinline__ int parts_of(const DecodeLaunch& a, int tiles) {
  return min((tiles + a.tiles_per_split - 1) / a.tiles_per_split, a.nsplit);
}

// head g of a (sequence, KV head): o of four channels from c4 on, the largest logit (unscaled), the sum
template <bool BF16>
__device__ __forceinline__ void store_row(const DecodeLaunch& a, int64_t row, int c4, float4 o, float mx, float l) {
  *reinterpret_cast<float4*>(a.out_o32 + row * kHeadDim + c4) = o;
  if (a.out_o)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out_o) + row * kHeadDim + c4) =
        make_uint2(pack2<BF16>(o.x, o.y), pack2<BF16>(o.z, o.w));
  if (c4 == 0) {
    a.out_m[row] = mx * kSoftmaxScale;
    a.out_l[row] = l;
  }
}

struct DecodeLds {
  float o[NW][16][kHeadDim + 4];
  float m[NW][16], l[NW][16];
};

template <bool BF16, bool E4M3, int SHAPE = 0>
__global__ __launch_bounds__(NW * kWave) void decode_kernel(const DecodeLaunch a) {
  __shared__ __align__(16) DecodeLds S;
  const int t = threadIdx.x, lane = lane_id(), w = __builtin_amdgcn_readfirstlane(t / kWave);
  const int j = lane >> 4, n = lane & 15;
  const int h = blockIdx.y, s = blockIdx.z;
  // (workgroups go to the XCDs in turn: without the shift the first parts, all that short sequences have,
  // would fall on one XCD where nsplit is a multiple of 8)
  const int part = (int)(blockIdx.x + h + s) % a.nsplit;
  const int G = a.group;
  const float kNegInf = -__builtin_inff();
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  const int lo = first_key<SHAPE>(a, s, kv);
  const int tiles = key_tiles(a, s, h, lo, kv), parts = max(parts_of(a, tiles), 1);
  if (part >= parts) return;
  float slope = 0.0f;
  if constexpr (SHAPE & kShapeSlopes) slope = slope_of<SHAPE>(a.sh, h * G + min(n, G - 1));

  u32x4_t qf[4];
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + ((int64_t)(s * a.c.num_kv_heads + h) * G + min(n, G - 1)) * kHeadDim;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    qf[x] = *reinterpret_cast<const u32x4_t*>(q + (E4M3 ? 64 * (x >> 1) + 16 * j + 8 * (x & 1) : 32 * x + 8 * j));

  WaveState st;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) st.acc[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  st.mx = kNegInf;
  st.ref = kNoRef;
  st.l = 0.0f;
  st.top = 0;

  const int sh = a.c.page_shift - 4;  // log2 of the tiles of a page
  const int64_t head_row = (int64_t)h * a.c.max_pages * a.c.page_size;
  // tile w of the part's runs of NW tiles, every parts-th run
  const int step = parts * NW, first = part * NW + w;
  const int mine = (tiles - first + step - 1) / step;
  // the first cache row, the first token and the tokens of the wave's tile i; no tokens: there is no such tile
  const auto find = [&](int i, int64_t& row, int& tok0, int& valid) {
    row = 0;
    tok0 = 0;
    valid = 0;
    if (i >= mine) return;
    const int x = first + step * i + (SHAPE && !a.pages ? lo / kTile : 0);
    const int sub = x & ((1 << sh) - 1);
    int lp = x >> sh;
    if (a.pages) lp = a.pages[((size_t)s * a.c.num_kv_heads + h) * a.cap + lp];
    const int64_t tok = ((int64_t)lp << a.c.page_shift) + sub * kTile;
    if (lp < 0 || tok >= kv || (SHAPE && (tok + kTile <= lo || lo >= kv))) return;
    const int phys = phys_page(a.b.page_table, a.b.table_stride, a.c.max_pages, s, lp);
    if (phys < 0) return;
    valid = (int)min(kv - tok, (int64_t)kTile);
    tok0 = (int)tok;
    row = head_row + ((int64_t)phys << a.c.page_shift) + sub * kTile;
  };
  for (int i0 = 0; i0 < mine; i0 += kWave) {
    // where the wave's next 64 tiles lie: lane i looks tile i0 + i up
    int64_t my_row;
    int my_tok, my_valid;
    find(i0 + lane, my_row, my_tok, my_valid);
    // the valid tiles, in order, the next one's loads ahead of a tile's products
    uint64_t todo = __ballot(my_valid > 0);
    if (!todo) continue;
    const auto take = [&](int& valid, int& tok, int64_t& row) {
      const int i = __builtin_ctzll(todo);
      todo &= todo - 1;
      valid = __builtin_amdgcn_readlane(my_valid, i);
      if constexpr (SHAPE) tok = __builtin_amdgcn_readlane(my_tok, i);
      row = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(my_row >> 32), i) << 32) |
                      (uint32_t)__builtin_amdgcn_readlane((int)my_row, i));
    };
    constexpr int NB = 2;  // tiles in flight per wave
    TileData<E4M3> d[NB];
    int valid[NB], tok[NB] = {0, 0};
    const auto skip_of = [&](int tok0) { return SHAPE ? max(lo - tok0, 0) : 0; };
    const auto next = [&](int x) {
      valid[x] = 0;
      if (!todo) return;
      int64_t row;
      take(valid[x], tok[x], row);
      load_tile<E4M3>(a.c, row, skip_of(tok[x]), valid[x], d[x]);
    };
#pragma unroll
    for (int x = 0; x < NB; ++x) next(x);
    while (valid[0]) {
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        if (!valid[x]) break;
        attend_tile<BF16, E4M3, SHAPE>(d[x], qf, skip_of(tok[x]), valid[x], kv - 1 - tok[x], slope, a.sh, st);
        next(x);
      }
    }
  }

  const float l = sum_rows(st.l);
  // An infinite value meets weight terms of 0 and of the other sign and comes out as NaN.  Where there is a NaN (and
  // the weights are none) the channel is the sum of its values that are not finite, whatever their weights.
  if constexpr (!E4M3) {
    bool odd = false;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= st.acc[cb][i] != st.acc[cb][i];
    if (__any(odd && l == l)) {
      f32x4_t sum[8];
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) sum[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < mine; ++x) {
        int64_t row;
        int tok, valid;
        find(x, row, tok, valid);
        for (int r = SHAPE ? max(lo - tok, 0) : 0; r < valid; ++r) {
          const uint16_t* v = static_cast<const uint16_t*>(a.c.v) + (row + r) * kHeadDim + 32 * j;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const u32x4_t y = *reinterpret_cast<const u32x4_t*>(v + 8 * i);
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) {
              const uint32_t bits = (y[cb >> 1] >> (16 * (cb & 1))) & 0xffffu;
              if (non_finite<BF16>(bits)) sum[cb][i] += h2f<BF16>(bits);
            }
          }
        }
      }
#pragma unroll
      for (int cb = 0; cb < 8; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.acc[cb][i] = sum[cb][i] == 0.0f ? st.acc[cb][i] : sum[cb][i];
    }
  }

  // the wave's state, normalised
  const float norm = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  if constexpr (E4M3) {
    const int by = st.top - 127 - kHeadroom;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[cb][i] = ldexpf(st.acc[cb][i], by);
  }
  // l relative to the logit itself, not to its rounded product with the scale
  const float exact = l == 0.0f || l != l ? l : l * exp2_hw(-fmaf(st.mx, kSoftmaxScale2, -st.ref));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int c = 0; c < 8; c += 4) {
      const float4 o = make_float4(st.acc[c][i] * norm, st.acc[c + 1][i] * norm, st.acc[c + 2][i] * norm, st.acc[c + 3][i] * norm);
      *reinterpret_cast<float4*>(&S.o[w][n][32 * j + 8 * i + c]) = o;
    }
  }
  if (j == 0) {
    S.m[w][n] = l != l ? l : st.mx;  // (maxima pass over NaN: a state of NaN must not look empty)
    S.l[w][n] = exact;
  }
  __syncthreads();
  // 32 threads per head, four channels each
  const int c4 = (t & 31) * 4;
  for (int g = t >> 5; g < G; g += 2 * NW) {
    float mx = kNegInf;
#pragma unroll
    for (int x = 0; x < NW; ++x) mx = fmaxf(mx, S.m[x][g]);
    float sum = 0.0f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float m = S.m[x][g];
      const float f = m == kNegInf ? 0.0f : S.l[x][g] * exp2_hw((m - mx) * kSoftmaxScale2);
      if (f == 0.0f) continue;
      const float4 y = *reinterpret_cast<const float4*>(&S.o[x][g][c4]);
      sum += f;
      o.x += f * y.x;
      o.y += f * y.y;
      o.z += f * y.z;
      o.w += f * y.w;
    }
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.nsplit == 1) {
      store_row<BF16>(a, (int64_t)(s * a.c.num_kv_heads + h) * G + g, c4, o, mx, sum);
    } else {
      const int64_t at = ((int64_t)(s * a.c.num_kv_heads + h) * a.nsplit + part) * G + g;
      *reinterpret_cast<float4*>(a.part_o + at * kHeadDim + c4) = o;
      if (c4 == 0) {
        a.part_ml[2 * at] = sum != sum ? sum : mx;
        a.part_ml[2 * at + 1] = sum;
      }
    }
  }
}

// The parts of one query head of one sequence, 32 of the 128 channels: eight threads take a part (four
// channels each), 32 parts at a time; the first 128 parts' rows are loaded before their weights are
// known.
constexpr int kMergeEarly = 4;

template <bool BF16, int SHAPE = 0>
__global__ __launch_bounds__(256) void merge_parts_kernel(const DecodeLaunch a) {
  __shared__ float so[4][32], sl[4], sm[4];
  const int t = threadIdx.x, slot = t >> 3, w = t / kWave;
  const int g = blockIdx.x >> 2, c4 = (blockIdx.x & 3) * 32 + (t & 7) * 4, h = blockIdx.y, s = blockIdx.z;
  const float kNegInf = -__builtin_inff();
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  const int parts = parts_of(a, key_tiles(a, s, h, first_key<SHAPE>(a, s, kv), kv));
  const int64_t base = (int64_t)(s * a.c.num_kv_heads + h) * a.nsplit;
  const auto at = [&](int p) { return (base + p) * a.group + g; };
  float4 y[kMergeEarly];
  float2 ml[kMergeEarly];
#pragma unroll
  for (int x = 0; x < kMergeEarly; ++x) {
    const int p = slot + 32 * x;
    y[x] = make_float4(0.f, 0.f, 0.f, 0.f);
    ml[x] = make_float2(kNegInf, 0.f);
    if (p < parts) {
      ml[x] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at(p));
      y[x] = *reinterpret_cast<const float4*>(a.part_o + at(p) * kHeadDim + c4);
    }
  }
  float mx = kNegInf;
#pragma unroll
  for (int x = 0; x < kMergeEarly; ++x) mx = fmaxf(mx, ml[x].x);
  for (int p = 32 * kMergeEarly + t; p < parts; p += 256) mx = fmaxf(mx, a.part_ml[2 * at(p)]);
  mx = wave_max(mx);
  if (lane_id() == 0) sm[w] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  float sum = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](const float2& st, const float4& v) {
    const float f = st.x == kNegInf ? 0.0f : st.y * exp2_hw((st.x - mx) * kSoftmaxScale2);
    if (f != 0.0f) {
      sum += f;
      o.x += f * v.x;
      o.y += f * v.y;
      o.z += f * v.z;
      o.w += f * v.w;
    }
  };
#pragma unroll
  for (int x = 0; x < kMergeEarly; ++x) add(ml[x], y[x]);
  for (int p = slot + 32 * kMergeEarly; p < parts; p += 32)
    add(*reinterpret_cast<const float2*>(a.part_ml + 2 * at(p)),
        *reinterpret_cast<const float4*>(a.part_o + at(p) * kHeadDim + c4));
  // the eight parts of a wave (lanes 8 apart), then the four waves
#pragma unroll
  for (int x = 8; x < kWave; x *= 2) {
    sum += __shfl_xor(sum, x);
    o.x += __shfl_xor(o.x, x);
    o.y += __shfl_xor(o.y, x);
    o.z += __shfl_xor(o.z, x);
    o.w += __shfl_xor(o.w, x);
  }
  if (lane_id() < 8) {
    *reinterpret_cast<float4*>(&so[w][4 * lane_id()]) = o;
    sl[w] = sum;
  }
  __syncthreads();
  if (t >= 8) return;
  sum = (sl[0] + sl[1]) + (sl[2] + sl[3]);
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = ((so[0][4 * t + i] + so[1][4 * t + i]) + (so[2][4 * t + i] + so[3][4 * t + i])) * inv;
  store_row<BF16>(a, (int64_t)(s * a.c.num_kv_heads + h) * a.group + g, c4, make_float4(r[0], r[1], r[2], r[3]), mx, sum);
}

template <bool BF16, int SHAPE>
const void* decode_fn(bool e4m3) {
  return e4m3 ? (const void*)decode_kernel<BF16, true, SHAPE> : (const void*)decode_kernel<BF16, false, SHAPE>;
}

}  // namespace

}  // namespace prr

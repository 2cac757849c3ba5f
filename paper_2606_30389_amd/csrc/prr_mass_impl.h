// The attention weight that cached tokens receive from new tokens.
#pragma once

#include <type_traits>

#include "prr_context.h"
#include "prr_shape.h"

namespace prr {

namespace {

// mass[j] = decay before[j] + sum over (token, query head) rows of exp(z_j - m) / l, with m and l of the attention that the
// rows have had.  With log2(l) in the exponent a weight is one multiply-add and one exponential of a logit (off by 4.0e-7 for 32
// tokens over 131072, where a division by l is off by 1.3e-7).
//
// A workgroup of four waves takes 64 KB keys of one sequence and KV head, a wave 16 KB of them, which stay in registers, and
// walks over the rows that see any of them, 64 at a time through LDS (two buffers, the next rows' loads in flight during a
// tile's products).  Lane 16j+n of a 16x16x32 product has row n's logits of keys 4j..4j+3 and adds its weights up by
// itself; lanes are joined once, at the end.  So no weight moves, and the order of every sum is fixed: parts of the rows are
// other workgroups' and are added by mass_join_kernel.
//
// Bound by the SIMDs: their matrix and vector instructions hardly overlap (256 cycles of products and 271 of multiply-adds,
// exponentials and additions, what 16 rows x 64 keys take, are 468 together at two waves a SIMD, 428 at four).  8191 tokens of
// float16, 32 / 8 heads, 315 us without a cap, 0.88 PFLOP/s, and 425 to 465 with one, e4m3 keys 3% more (with a cap and slopes
// their four blocks take all 256 registers and spill 2); 32 tokens over 131072, 32 / 2 heads, 49 to 58 us, of which 13 are the
// keys'.  32x32x16 products overlap better (390) but leave no registers for the next rows'
// products under these rows' weights: 7% slower; three waves a SIMD spill, 25% slower; two blocks a wave 3 to 9%.
//
// Every 32 tiles a lane's sums go to a second set, so that a sum of n rows is off by about (128 + n / 2048) 2^-24 at most.
constexpr int kRows = 64;                 // rows of a tile
constexpr int kFlush = 32;

template <bool BF16>
__device__ __forceinline__ f32x4_t mass_mfma(const u32x4_t& a, const u32x4_t& b, f32x4_t c) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  }
}

// Row r (of `rows`, G a token) of the counted tokens: its token and head
__device__ __forceinline__ int mass_over_group(int x, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)x, magic) : x; }

template <bool BF16, bool E4M3, int KB, int SHAPE>
__global__ __launch_bounds__(256, 2) void mass_kernel(const MassLaunch a) {
  __shared__ __align__(16) uint16_t lq[2][kRows * kHeadDim];
  __shared__ float l_total[KB][4][256];
  __shared__ float l_ref[2][kRows], l_slope[2][kRows];
  __shared__ int l_lo[2][kRows], l_hi[2][kRows], l_pos[2][kRows];
  __shared__ int l_none[2];  // whether a row of the tile gives no weight (1% of 8191 tokens' time)
  const int t = threadIdx.x, lane = lane_id(), w = __builtin_amdgcn_readfirstlane(t / kWave);
  const int j = lane >> 4, n = lane & 15;
  // (the heads of a group of keys side by side: the first keys, which most rows see, of all heads begin first)
  const int h = (int)(blockIdx.x % a.c.num_kv_heads), s = blockIdx.z, G = a.group;
  const int step = a.nsplit * a.c.num_kv_heads;
  const Seq sq = seq_at(a.b, s);
  const int q_len = sq.q1 - sq.q0, counted = a.last ? min(a.last, q_len) : q_len;
  const int first = sq.kv - q_len;  // position of the first new token
  const int prefix = a.sh.prefix ? min(a.sh.prefix[s], sq.kv) : 0;
  const int list = a.pages ? min(max(a.page_count[(size_t)s * a.c.num_kv_heads + h], 0), a.cap) : 0;
  const int64_t keys = a.pages ? (int64_t)list << a.c.page_shift : sq.kv;
  const int64_t head_row = (int64_t)h * a.c.max_pages * a.c.page_size;

  for (int kg = (int)(blockIdx.x / step); (int64_t)kg * 64 * KB < keys; kg += (int)(gridDim.x / step)) {
    // (turned from group to group, as workgroups go to the XCDs in turn and a group's first part has the diagonal)
    const int part = (int)((blockIdx.x / a.c.num_kv_heads + kg) % a.nsplit);
    // the wave's blocks of 16 keys: first cache row, position of the first key, keys that there are
    int64_t my_row = 0;
    int my_tok = 0, my_valid = 0;
    if (lane < KB) {
      const int64_t x = ((int64_t)kg * 4 * KB + w * KB + lane) * 16;
      if (x < keys) {
        int lp = (int)(x >> a.c.page_shift);
        const int off = (int)(x & (a.c.page_size - 1));
        if (a.pages) lp = a.pages[((size_t)s * a.c.num_kv_heads + h) * a.cap + lp];
        const int64_t tok = ((int64_t)lp << a.c.page_shift) + off;
        const int phys = lp >= 0 && tok < sq.kv ? phys_page(a.b.page_table, a.b.table_stride, a.c.max_pages, s, lp) : -1;
        if (phys >= 0) {
          my_row = head_row + ((int64_t)phys << a.c.page_shift) + off;
          my_tok = (int)tok;
          my_valid = (int)min(sq.kv - tok, (int64_t)16);
        }
      }
    }
    int64_t row0[KB];
    int tok0[KB], valid[KB];
    u32x4_t kf[KB][4];
    float ks[KB][4];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      row0[b] = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(my_row >> 32), b) << 32) |
                          (uint32_t)__builtin_amdgcn_readlane((int)my_row, b));
      tok0[b] = __builtin_amdgcn_readlane(my_tok, b);
      valid[b] = __builtin_amdgcn_readlane(my_valid, b);
      // (rows behind the last repeat it; a block that is not there reads row 0 of the head)
      const int64_t r = row0[b] + max(min(n, valid[b] - 1), 0);
      if constexpr (E4M3) {
        const uint8_t* k = static_cast<const uint8_t*>(a.c.k) + (valid[b] ? r : head_row) * kHeadDim + 16 * j;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const u32x4_t c = *reinterpret_cast<const u32x4_t*>(k + 64 * x);
          kf[b][2 * x] = u32x4_t{unpack_codes<BF16, false>(c[0], 1.0f), unpack_codes<BF16, true>(c[0], 1.0f),
                                 unpack_codes<BF16, false>(c[1], 1.0f), unpack_codes<BF16, true>(c[1], 1.0f)};
          kf[b][2 * x + 1] = u32x4_t{unpack_codes<BF16, false>(c[2], 1.0f), unpack_codes<BF16, true>(c[2], 1.0f),
                                     unpack_codes<BF16, false>(c[3], 1.0f), unpack_codes<BF16, true>(c[3], 1.0f)};
        }
        const uint32_t sc = *reinterpret_cast<const uint32_t*>(a.c.k_scale + (valid[b] ? row0[b] : head_row) + 4 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) ks[b][i] = __uint_as_float(((sc >> (8 * i)) & 0xffu) << 23);
      } else {
        const uint16_t* k = static_cast<const uint16_t*>(a.c.k) + (valid[b] ? r : head_row) * kHeadDim + 8 * j;
#pragma unroll
        for (int x = 0; x < 4; ++x) kf[b][x] = *reinterpret_cast<const u32x4_t*>(k + 32 * x);
      }
    }
    // positions of the wave's keys, and of the workgroup's (without lists they follow each other)
    int wk0 = 0x7fffffff, wk1 = 0;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if (!valid[b]) continue;
      wk0 = min(wk0, tok0[b]);
      wk1 = max(wk1, tok0[b] + valid[b]);
    }
    const bool run = !a.pages;  // the wave's keys are [wk0, wk1)
    // the counted tokens that may see any of them
    int i0 = max(q_len - counted, -first), i1 = q_len;
    if (!a.pages) {
      const int g0 = kg * 64 * KB, g1 = (int)min((int64_t)g0 + 64 * KB, keys);
      if (prefix <= g0) i0 = max(i0, g0 - first);
      if (a.sh.window) i1 = (int)max(min((int64_t)i1, (int64_t)g1 + a.sh.window - 1 - first), (int64_t)0);
    }
    if (a.sh.first && !a.pages) {  // (documents: the first and the last token that see a key of the workgroup's)
      const int g0 = kg * 64 * KB, g1 = (int)min((int64_t)g0 + 64 * KB, keys);
      int lo = 0x7fffffff, hi = 0;
      for (int i = i0 + t; i < i1; i += 256) {
        const Span sp = span_at(a.sh.window, a.sh.first[sq.q0 + i], prefix, first + i, sq.kv);
        if (sp.lo < min(sp.hi, g1) && sp.hi > g0) {
          lo = min(lo, i);
          hi = i + 1;
        }
      }
      lo = (int)wave_umin((uint32_t)lo);
      hi = (int)wave_umax((uint32_t)hi);
      if (lane == 0) {
        l_lo[0][w] = lo;
        l_hi[0][w] = hi;
      }
      __syncthreads();
      i0 = min(min(l_lo[0][0], l_lo[0][1]), min(l_lo[0][2], l_lo[0][3]));
      i1 = max(max(l_hi[0][0], l_hi[0][1]), max(l_hi[0][2], l_hi[0][3]));
      __syncthreads();
    }
    const int rows = max(i1 - i0, 0) * G, tiles = (rows + kRows - 1) / kRows;
    const int per = (tiles + a.nsplit - 1) / a.nsplit;
    const int t0 = min(part * per, tiles), t1 = min(t0 + per, tiles);

    f32x4_t sum[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) sum[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const bool flushes = t1 - t0 > kFlush;
    if (flushes) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) l_total[b][i][t] = 0.0f;
    }

    // Thread t brings 16 bytes of rows t/16 + 16 x; the place of row r's 16 bytes c is c ^ (r % 16), so that a read of the
    // same bytes of 16 rows meets every bank once.  Threads 0..63 bring what is known of row t.  Nothing of it is looked at
    // before the products of the tile before are done.  A row lies at an offset from the tile's first token that is the same
    // in every tile where the group size divides 64.
    u32x4_t qr[4];
    uint32_t offset[4], info = 0;  // bytes; rows of m and l
    float r_m = 0.0f, r_l = 0.0f, r_slope = 0.0f;
    int r_first = 0, r_tok = 0, r_pos = 0;
    bool r_live = false;
    const bool aligned = (G & (G - 1)) == 0;
    const int heads = a.c.num_kv_heads * G;
    const auto tile_token = [&](int tile) { return mass_over_group(tile * kRows, a.magic); };
    const auto load = [&](int tile, bool find) {
      const int r0 = tile * kRows, tok0 = tile_token(tile), h0 = r0 - tok0 * G;
      if (find || !aligned || r0 + kRows > rows) {
        const auto at = [&](int local, int& tok, int& head) {
          const int r = h0 + min(local, rows - 1 - r0);
          tok = mass_over_group(r, a.magic);
          head = r - tok * G;
          return (uint32_t)(tok * heads + head);
        };
        int tok, head;
#pragma unroll
        for (int x = 0; x < 4; ++x) offset[x] = at((t >> 4) + 16 * x, tok, head) * (2 * kHeadDim) + 16 * (t & 15);
        if (t < kRows) {
          info = at(t, r_tok, head);
          if constexpr (SHAPE & kShapeSlopes) r_slope = slope_of<SHAPE>(a.sh, h * G + head);
        }
      }
      const int64_t row = ((int64_t)(sq.q0 + i0 + tok0) * a.c.num_kv_heads + h) * G;
      const char* const q = static_cast<const char*>(a.q) + row * (2 * kHeadDim);
#pragma unroll
      for (int x = 0; x < 4; ++x) qr[x] = *reinterpret_cast<const u32x4_t*>(q + offset[x]);
      if (t < kRows) {
        r_m = (a.m + row)[info];
        r_l = (a.l + row)[info];
        r_first = a.sh.first ? (a.sh.first + sq.q0 + i0 + tok0)[r_tok] : 0;
        r_pos = first + i0 + tok0 + r_tok;
        r_live = r0 + t < rows;  // (rows behind the last see nothing)
      }
    };
    // Whether the wave's keys are seen by every row of a tile, as far as that is known without looking at the rows
    const auto known_whole = [&](int tile) {
      if (!run || a.sh.first || (tile + 1) * kRows > rows || wk1 == 0) return false;
      const int p0 = first + i0 + tile_token(tile), p1 = first + i0 + mass_over_group(tile * kRows + kRows - 1, a.magic);
      return max(p0 + 1, prefix) >= wk1 && (!a.sh.window || p1 - a.sh.window + 1 <= wk0);
    };
    const auto store = [&](int buf) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<u32x4_t*>(&lq[buf][((t >> 4) + 16 * x) * kHeadDim + 8 * ((t & 15) ^ ((t >> 4) & 15))]) = qr[x];
      if (t < kRows) {
        const Span sp = span_at(a.sh.window, r_first, prefix, r_pos, sq.kv);
        l_ref[buf][t] = r_l == 0.0f ? __builtin_inff() : fmaf(r_m, kLog2e, __builtin_amdgcn_logf(r_l));
        l_lo[buf][t] = sp.lo;
        l_hi[buf][t] = r_live && r_l != 0.0f ? sp.hi : sp.lo;  // (a row of l = 0 may hold anything: it is hidden as one behind the last)
        const bool none = __any(r_l == 0.0f);
        if (t == 0) l_none[buf] = none;
        if constexpr (SHAPE & kShapeSlopes) {
          l_pos[buf][t] = r_pos;
          l_slope[buf][t] = r_slope;
        }
      }
    };
    // 16 rows, from row 16 u of the tile in the buffer on
    const auto products = [&](int buf, int u, auto masked) {
      u32x4_t qf[4];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        qf[x] = *reinterpret_cast<const u32x4_t*>(&lq[buf][(16 * u + n) * kHeadDim + 8 * ((E4M3 ? 8 * (x >> 1) + 2 * j + (x & 1) : 4 * x + j) ^ n)]);
      const float ref = l_ref[buf][16 * u + n];
      f32x4_t d[KB];
#pragma unroll
      for (int b = 0; b < KB; ++b) d[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int b = 0; b < KB; ++b) d[b] = mass_mfma<BF16>(kf[b][x], qf[x], d[b]);
      if constexpr (E4M3) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[b][i] *= ks[b][i];
      }
      [[maybe_unused]] bool small = false;
      if constexpr (SHAPE & kShapeCap) {
        float most = 0.0f;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(d[b][i]));
        small = __all(most < a.sh.small);
        if constexpr (SHAPE & kShapeSlopes) {
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[b][i] = cap_wide(d[b][i], a.sh);
        }
      }
      if constexpr (SHAPE & kShapeSlopes) {
        const int pos = l_pos[buf][16 * u + n];
        const float slope = l_slope[buf][16 * u + n];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
          const float ahead = (float)(tok0[b] + 4 * j - pos);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[b][i] = fmaf(-slope, fabsf(ahead + (float)i), d[b][i]);
        }
      }
      if constexpr (SHAPE == kShapeCap) {
        if (small) {
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[b][i] = exp2_hw(cap_exponent(d[b][i], ref, kSoftmaxScale2, true, a.sh));
        } else {
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[b][i] = exp2_hw(cap_exponent(d[b][i], ref, kSoftmaxScale2, false, a.sh));
        }
      } else {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[b][i] = exp2_hw(fmaf(d[b][i], kSoftmaxScale2, -ref));
      }
      if constexpr (masked.value) {
        const int lo = l_lo[buf][16 * u + n], hi = l_hi[buf][16 * u + n];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
          const uint32_t at = (uint32_t)(tok0[b] + 4 * j - lo), seen = (uint32_t)(hi - lo);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[b][i] = at + (uint32_t)i < seen ? d[b][i] : 0.0f;
        }
      }
#pragma unroll
      for (int b = 0; b < KB; ++b) sum[b] += d[b];
    };
    // The tile in the buffer: a lane looks at a row's keys
    const auto tile_products = [&](int tile, int buf, int none) {
      if (known_whole(tile) && !__builtin_amdgcn_readfirstlane(none)) {
#pragma unroll
        for (int u = 0; u < kRows / 16; ++u) products(buf, u, std::false_type{});
        return;
      }
      const int lo = l_lo[buf][lane], hi = l_hi[buf][lane];
      const uint64_t some = __ballot(lo < wk1 && hi > wk0 && lo < hi);
      const uint64_t whole = run ? __ballot(lo <= wk0 && hi >= wk1) : 0;
      for (int u = 0; u < kRows / 16; ++u) {
        if (((whole >> (16 * u)) & 0xffff) == 0xffff) {
          products(buf, u, std::false_type{});
        } else if ((some >> (16 * u)) & 0xffff) {
          products(buf, u, std::true_type{});
        }
      }
    };

    if (t0 < t1) {
      load(t0, true);
      store(0);
      __syncthreads();
      for (int tile = t0; tile < t1; ++tile) {
        const int buf = (tile - t0) & 1;
        const int none = l_none[buf];  // (on its way during the loads)
        if (tile + 1 < t1) load(tile + 1, false);
        tile_products(tile, buf, none);
        if (tile + 1 < t1) store(buf ^ 1);
        if (flushes && ((tile - t0) & (kFlush - 1)) == kFlush - 1) {
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              l_total[b][i][t] += sum[b][i];
              sum[b][i] = 0.0f;
            }
        }
        __syncthreads();
      }
    }
    if (flushes) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[b][i] += l_total[b][i][t];
    }

#pragma unroll
    for (int b = 0; b < KB; ++b) {
      float r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = sum16(sum[b][i]);
      if (n < 4) {  // lane 16j+i stores key 4j+i
        const float v = n == 0 ? r[0] : n == 1 ? r[1] : n == 2 ? r[2] : r[3];
        if (a.nsplit > 1) {
          const int64_t unit = ((int64_t)part * a.b.n_seqs + s) * a.c.num_kv_heads + h;
          a.part[unit * a.part_keys + ((int64_t)kg * 4 * KB + w * KB + b) * 16 + 4 * j + n] = v;
        } else if (4 * j + n < valid[b]) {
          const int64_t at = row0[b] + 4 * j + n;
          a.mass[at] = a.before ? fmaf(a.decay, a.before[at], v) : v;
        }
      }
    }
  }
}

template <bool BF16, bool E4M3, int KB>
const void* mass_fn(int shape) {
  switch (shape & (kShapeCap | kShapeSlopes)) {
    case 0: return (const void*)mass_kernel<BF16, E4M3, KB, 0>;
    case kShapeCap: return (const void*)mass_kernel<BF16, E4M3, KB, kShapeCap>;
    case kShapeSlopes: return (const void*)mass_kernel<BF16, E4M3, KB, kShapeSlopes>;
    default: return (const void*)mass_kernel<BF16, E4M3, KB, kShapeCap | kShapeSlopes>;
  }
}

template <bool BF16>
const void* mass_fn_of(const MassLaunch& a) {
  if (a.e4m3) return a.blocks == 4 ? mass_fn<BF16, true, 4>(a.shape) : mass_fn<BF16, true, 1>(a.shape);
  return a.blocks == 4 ? mass_fn<BF16, false, 4>(a.shape) : mass_fn<BF16, false, 1>(a.shape);
}

}  // namespace

}  // namespace prr

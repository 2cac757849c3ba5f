// Rotary positions with the cache write, and an e4m3 cache read back.
#include "prr_context.h"

namespace prr {

namespace {

// =====================================================================================
// rotary positions, keys and values into the cache
// =====================================================================================
// A wave holds one token; 16 lanes hold one head's row, 8 channels each, so a wave takes four rows
// (queries, then keys, then values) at a time.  Lane u < rot/8 of a row holds four pairs: channels
// 8u..8u+7 (interleaved), or 4u..4u+3 and rot/2+4u.. (halves); either way its pairs are 4u..4u+3, so
// no lane needs another's channels, and the four angles are formed once for all rows of the token.
// Other lanes hold 8 plain channels.  An angle is reduced in float64 to a fraction of a turn (a
// position of 2^30 keeps 20 bits behind the point of a turn), the rest is float32.
//
// Bound by memory: 32768 tokens of 32 / 2 heads in 116 us, 5.2 TB/s of what has to be read and written,
// the rate of a large copy.
template <bool BF16, bool E4M3, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_append_kernel(const RopeLaunch a) {
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  const int t = wave / a.splits, part = wave - t * a.splits;
  const BatchArgs& b = a.b;
  if (t >= (b.cu_q ? min(b.cu_q[b.n_seqs], b.total_q) : b.n_seqs)) return;
  // the last sequence that starts at or before row t, 64 candidates at a time
  int s = t;
  if (b.cu_q) {
    s = 0;
    for (int n = b.n_seqs; n > 1;) {
      const int step = (n + kWave - 1) / kWave;
      const bool ok = lane * step < n && b.cu_q[s + lane * step] <= t;
      const int at = max(__popcll(__ballot(ok)) - 1, 0) * step;
      s += at;
      n = min(step, n - at);
    }
  }
  const Seq sq = seq_at(b, s);
  const int pos = sq.kv - (sq.q1 - sq.q0) + (t - sq.q0);
  const int lp = pos >> a.c.page_shift;
  const int phys = pos >= 0 && pos < sq.kv ? phys_page(b.page_table, b.table_stride, a.c.max_pages, s, lp) : -1;
  const int off = pos & (a.c.page_size - 1);

  const int u = lane & 15, slot = lane >> 4;
  const bool rotated = u < a.rot_dim / 8;
  int ca = 8 * u, cb = 8 * u + 4;  // channels of the lane's two groups of four
  if (!INTERLEAVED && rotated) {
    ca = 4 * u;
    cb = a.rot_dim / 2 + 4 * u;
  }
  float cs[4], sn[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) cs[i] = sn[i] = 0.0f;
  if (rotated) {
    const double p = (double)(a.positions ? a.positions[t] : pos) * 0.15915494309189535;  // 1/2pi
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double turns = p * a.freqs[4 * u + i];
      float si, co;
      sincospif(2.0f * (float)(turns - rint(turns)), &si, &co);
      cs[i] = co * a.scale;
      sn[i] = si * a.scale;
    }
  }

  const int hq = a.q ? a.num_q_heads : 0, hkv = a.k ? a.c.num_kv_heads : 0;
  const int rows = hq + 2 * hkv;
  for (int r = 4 * part + slot; r < rows; r += 4 * a.splits) {
    const bool is_q = r < hq, is_v = r >= hq + hkv;
    const int head = is_q ? r : is_v ? r - hq - hkv : r - hq;
    const uint16_t* src = static_cast<const uint16_t*>(is_q ? a.q : is_v ? a.v : a.k) +
                          (int64_t)t * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + head * kHeadDim;
    const uint2 wa = *reinterpret_cast<const uint2*>(src + ca), wb = *reinterpret_cast<const uint2*>(src + cb);
    float x[8] = {h2f<BF16>(wa.x & 0xffffu), h2f<BF16>(wa.x >> 16), h2f<BF16>(wa.y & 0xffffu), h2f<BF16>(wa.y >> 16),
                  h2f<BF16>(wb.x & 0xffffu), h2f<BF16>(wb.x >> 16), h2f<BF16>(wb.y & 0xffffu), h2f<BF16>(wb.y >> 16)};
    if (rotated && !is_v) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : i + 4;
        const float xa = x[ia], xb = x[ib];
        x[ia] = xa * cs[i] - xb * sn[i];
        x[ib] = xa * sn[i] + xb * cs[i];
      }
    }
    if (is_q || !E4M3) {
      if (!is_q && phys < 0) continue;
      uint16_t* dst = is_q ? static_cast<uint16_t*>(a.q_out) + ((int64_t)t * hq + head) * kHeadDim
                           : static_cast<uint16_t*>(is_v ? a.c.v : a.c.k) +
                                 (((int64_t)head * a.c.max_pages + phys) * a.c.page_size + off) * kHeadDim;
      *reinterpret_cast<uint2*>(dst + ca) = make_uint2(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]));
      *reinterpret_cast<uint2*>(dst + cb) = make_uint2(pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
    } else {
      // 2^e from the exponent and mantissa of the row's largest magnitude: 448 = 1.75 * 2^8
      constexpr float kLimit = BF16 ? 0.9375f * 0x1p127f * 2.0f : 0.9375f * 0x1p16f;
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fminf(fmaxf(x[i], -kLimit), kLimit);
        x[i] = x[i] == x[i] ? y : x[i];
        top = fmaxf(top, fabsf(x[i]));  // (fmaxf passes over NaN)
      }
      top = max16(top);
      const uint32_t bits = __float_as_uint(top);
      const int e = max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
      if (phys < 0) continue;
      const int64_t row = ((int64_t)head * a.c.max_pages + phys) * a.c.page_size + off;
      uint8_t* dst = static_cast<uint8_t*>(is_v ? a.c.v : a.c.k) + row * kHeadDim;
      int lo = 0, hi = 0;
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, lo, false);
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, hi, false);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, hi, true);
      *reinterpret_cast<int*>(dst + ca) = lo;
      *reinterpret_cast<int*>(dst + cb) = hi;
      if (u == 0) (is_v ? a.c.v_scale : a.c.k_scale)[row] = (uint8_t)(e + 127);
    }
  }
}

template <bool BF16, bool E4M3>
hipError_t launch_rope(const RopeLaunch& a, int blocks, hipStream_t stream) {
  const void* f = a.interleaved ? (const void*)rope_append_kernel<BF16, E4M3, true>
                                : (const void*)rope_append_kernel<BF16, E4M3, false>;
  return launch_one(f, dim3(blocks), 256, stream, a);
}

// =====================================================================================
// an e4m3 cache's pages in 16 bits
// =====================================================================================
// Eight lanes per row, 16 codes each: one 16-byte load, two 16-byte stores.  The conversion multiplies by the
// power of two and rounds once (exact but for subnormal results).  Bound by memory: 131072 tokens of two KV
// heads in 39 us, 5.2 TB/s.
template <bool BF16>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheReadLaunch a) {
  const int64_t per_head = (int64_t)a.pages << a.c.page_shift, total = per_head * a.c.num_kv_heads * 8;
  const bool is_v = blockIdx.y != 0;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
    const int64_t row = x >> 3;
    const int c16 = (int)(x & 7) * 16;
    const int h = (int)(row / per_head);
    const int64_t in_head = row - h * per_head;
    const int lp = a.page_begin + (int)(in_head >> a.c.page_shift), off = (int)in_head & (a.c.page_size - 1);
    if (((int64_t)lp << a.c.page_shift) + off >= a.num_tokens) continue;
    const int phys = phys_page(a.page_table, 0x7fffffff, a.c.max_pages, 0, lp);
    if (phys < 0) continue;
    const int64_t from = ((int64_t)h * a.c.max_pages + phys) * a.c.page_size + off;
    const uint4 w =
        *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? a.c.v : a.c.k) + from * kHeadDim + c16);
    const uint32_t byte = (is_v ? a.c.v_scale : a.c.k_scale)[from];
    const float scale = __uint_as_float(byte << 23);
    uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(is_v ? a.v_out : a.k_out) + row * kHeadDim + c16);
    dst[0] = make_uint4(unpack_codes<BF16, false>(w.x, scale), unpack_codes<BF16, true>(w.x, scale),
                        unpack_codes<BF16, false>(w.y, scale), unpack_codes<BF16, true>(w.y, scale));
    dst[1] = make_uint4(unpack_codes<BF16, false>(w.z, scale), unpack_codes<BF16, true>(w.z, scale),
                        unpack_codes<BF16, false>(w.w, scale), unpack_codes<BF16, true>(w.w, scale));
  }
}

}  // namespace

hipError_t launch_rope_append(RopeLaunch a, hipStream_t stream) {
  const int rows = (a.q ? a.num_q_heads : 0) + (a.k ? 2 * a.c.num_kv_heads : 0);
  const int tokens = a.b.cu_q ? a.b.total_q : a.b.n_seqs;
  // one wave per token forms its angles once (32768 tokens, 32 / 2 heads: 116 us, 173 with nine waves a
  // token); few tokens spread their rows over more waves, up to two per SIMD of the chip (one token 2.8 us,
  // 4.8 by one wave; 64 tokens of 32 / 8 heads 3.8, 7.9)
  a.splits = (int)min((int64_t)(rows + 3) / 4, max((int64_t)1, (int64_t)2048 / tokens));
  const int64_t waves = (int64_t)tokens * a.splits;
  const int blocks = (int)((waves + 3) / 4);
  if (a.bf16) return a.e4m3 ? launch_rope<true, true>(a, blocks, stream) : launch_rope<true, false>(a, blocks, stream);
  return a.e4m3 ? launch_rope<false, true>(a, blocks, stream) : launch_rope<false, false>(a, blocks, stream);
}

hipError_t launch_cache_read(const CacheReadLaunch& a, hipStream_t stream) {
  const int64_t blocks = (((int64_t)a.c.num_kv_heads * a.pages << a.c.page_shift) * 8 + 255) / 256;
  const dim3 grid((unsigned)min(blocks, (int64_t)1 << 22), 2);
  return launch_one(a.bf16 ? (const void*)cache_read_kernel<true> : (const void*)cache_read_kernel<false>, grid, 256, stream, a);
}

}  // namespace prr

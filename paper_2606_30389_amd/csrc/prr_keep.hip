// Which tokens of a cache are kept, and their rows to their new places.
#include "prr_context.h"

namespace prr {

namespace {

// =====================================================================================
// the tokens of the largest mass
// =====================================================================================
// Of a sequence and KV head: the first `sink` and the last `recent` tokens, and of those between them the ones of the largest
// mass, the lower position first among equals.  A mass becomes a 32-bit key of the same order; counting the keys by 11, 11
// and 10 bits finds the key of the last token taken, and how many of that key are.  Positions come out in order: a token's
// place is the number of taken tokens before it.
//
// Up to 32768 tokens one workgroup does all of it, the keys in registers; the counts lie in LDS eightfold, as masses
// share few exponents and lanes that count the same bin wait for each other.  More tokens are cut into chunks of as
// many workgroups, a launch per step: counts of each chunk in device memory, added up by all.
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 2048, kCopies = 8;
constexpr int kSmall = 32768;      // tokens of one workgroup
constexpr int kMaxChunks = 64;

// Larger mass, larger key; NaN below everything
__device__ __forceinline__ uint32_t mass_key(float f) { return f != f ? 0u : score_key(f); }

__device__ __forceinline__ uint32_t bin_of(uint32_t key, int level) {
  return level == 0 ? key >> 21 : level == 1 ? (key >> 10) & 2047u : key & 1023u;
}

struct Unit {
  int kv, count, sink, end;  // tokens; kept ones; [sink, end): those chosen by their mass
};
__device__ __forceinline__ Unit unit_of(const KeepLaunch& a, int s) {
  Unit u;
  u.kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  u.count = min(a.budget, u.kv);
  u.sink = u.count == u.kv ? u.kv : a.sink;
  u.end = u.count == u.kv ? u.kv : u.kv - a.recent;
  return u;
}

// The keys of tokens [p, p + 4), p a multiple of 4 and below kv; what is behind kv, or has no page, is 0
__device__ __forceinline__ void load_keys(const KeepLaunch& a, int s, int h, int p, int kv, uint32_t (&key)[4]) {
  const int phys = phys_page(a.b.page_table, a.b.table_stride, a.max_pages, s, p >> a.page_shift);
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (phys >= 0)
    v = *reinterpret_cast<const float4*>(a.mass + (((int64_t)h * a.max_pages + phys) << a.page_shift) + (p & (a.page_size - 1)));
  key[0] = phys >= 0 ? mass_key(v.x) : 0u;
  key[1] = phys >= 0 ? mass_key(v.y) : 0u;
  key[2] = phys >= 0 ? mass_key(v.z) : 0u;
  key[3] = phys >= 0 ? mass_key(v.w) : 0u;
}

// The bin that holds the need-th largest key, and how many of the bin's keys are taken; c0, c1: the thread's two bins'
// counts (bins 2 t, 2 t + 1).  need >= 1 and at most all of them.
__device__ __forceinline__ void find_bin(int c0, int c1, int need, int* wave_tot, int* found, int& bin, int& rest) {
  int all;
  const int before = block_exclusive_scan<kThreads>(c0 + c1, wave_tot, all);
  const int above1 = all - before - c0 - c1, above0 = above1 + c1;  // keys in higher bins
  const int t = threadIdx.x;
  if (above1 < need && need <= above1 + c1) {
    found[0] = 2 * t + 1;
    found[1] = need - above1;
  }
  if (above0 < need && need <= above0 + c0) {
    found[0] = 2 * t;
    found[1] = need - above0;
  }
  __syncthreads();
  bin = found[0];
  rest = found[1];
  __syncthreads();
}

struct Taken {
  uint32_t key;  // the threshold
  int ties;      // of its key, the first so many are taken
};
// Whether the token at p is kept for certain, and whether it is of the threshold's key
__device__ __forceinline__ void classify(const Unit& u, const Taken& tk, int p, uint32_t key, bool& gt, bool& tie) {
  const bool choice = p >= u.sink && p < u.end;
  gt = p < u.kv && (!choice || key > tk.key);
  tie = choice && key == tk.key;
}

template <int ITS>
__global__ __launch_bounds__(kThreads) void keep_kernel(const KeepLaunch a) {
  __shared__ uint32_t hist[kBins * kCopies];
  __shared__ int wave_tot[kWaves], found[2];
  __shared__ int tot_gt[ITS * kWaves], tot_tie[ITS * kWaves];
  const int t = threadIdx.x, lane = lane_id(), w = t / kWave;
  const int h = blockIdx.x, s = blockIdx.y;
  const Unit u = unit_of(a, s);
  if (t == 0 && h == 0) a.kept[s] = u.count;
  int32_t* const out = a.keep + ((int64_t)s * a.num_kv_heads + h) * a.budget;
  if (u.count == u.kv) {
    for (int p = t; p < u.count; p += kThreads) out[p] = p;
    return;
  }
  uint32_t key[ITS][4];
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    const int p = it * 4 * kThreads + 4 * t;
    key[it][0] = key[it][1] = key[it][2] = key[it][3] = 0u;
    if (p < u.kv) load_keys(a, s, h, p, u.kv, key[it]);
  }
  int need = u.count - u.sink - (u.kv - u.end);
  Taken tk = {0xffffffffu, 0};
  if (need > 0) {
    uint32_t prefix = 0;
    for (int level = 0; level < 3; ++level) {
      for (int x = t; x < kBins * kCopies; x += kThreads) hist[x] = 0;
      __syncthreads();
      const int shift = level == 0 ? 32 : level == 1 ? 21 : 10;
#pragma unroll
      for (int it = 0; it < ITS; ++it)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = it * 4 * kThreads + 4 * t + e;
          const bool in = p >= u.sink && p < u.end && (level == 0 || key[it][e] >> shift == prefix);
          if (in) atomicAdd(&hist[bin_of(key[it][e], level) * kCopies + (lane & (kCopies - 1))], 1u);
        }
      __syncthreads();
      int c0 = 0, c1 = 0;
#pragma unroll
      for (int x = 0; x < kCopies; ++x) {
        c0 += (int)hist[2 * t * kCopies + x];
        c1 += (int)hist[(2 * t + 1) * kCopies + x];
      }
      int bin, rest;
      find_bin(c0, c1, need, wave_tot, found, bin, rest);
      prefix = level == 0 ? (uint32_t)bin : (prefix << (level == 1 ? 11 : 10)) | (uint32_t)bin;
      need = rest;
    }
    tk.key = prefix;
    tk.ties = need;
  }
  // places: counts of each (step, wave), then within the wave
  int in_gt[ITS], in_tie[ITS];
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    int g = 0, e4 = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bool gt, tie;
      classify(u, tk, it * 4 * kThreads + 4 * t + e, key[it][e], gt, tie);
      g += gt;
      e4 += tie;
    }
    in_gt[it] = wave_inclusive_scan(g);
    in_tie[it] = wave_inclusive_scan(e4);
    if (lane == kWave - 1) {
      tot_gt[it * kWaves + w] = in_gt[it];
      tot_tie[it * kWaves + w] = in_tie[it];
    }
    in_gt[it] -= g;
    in_tie[it] -= e4;
  }
  __syncthreads();
  if (w == 0) {  // exclusive sums over the (step, wave)s, 64 at a time
    int base_g = 0, base_t = 0;
    for (int x = lane; x < (ITS * kWaves + kWave - 1) / kWave * kWave; x += kWave) {
      const int g = x < ITS * kWaves ? tot_gt[x] : 0, e4 = x < ITS * kWaves ? tot_tie[x] : 0;
      const int ig = wave_inclusive_scan(g), ie = wave_inclusive_scan(e4);
      if (x < ITS * kWaves) {
        tot_gt[x] = base_g + ig - g;
        tot_tie[x] = base_t + ie - e4;
      }
      base_g += __builtin_amdgcn_readlane(ig, kWave - 1);
      base_t += __builtin_amdgcn_readlane(ie, kWave - 1);
    }
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    int g = tot_gt[it * kWaves + w] + in_gt[it], e4 = tot_tie[it * kWaves + w] + in_tie[it];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = it * 4 * kThreads + 4 * t + e;
      bool gt, tie;
      classify(u, tk, p, key[it][e], gt, tie);
      const int at = g + min(e4, tk.ties);
      if ((gt || (tie && e4 < tk.ties)) && (uint32_t)at < (uint32_t)u.count) out[at] = p;
      g += gt;
      e4 += tie;
    }
  }
}

// -------------------------------------------------------------------------------------
// Several chunks.  Device memory of a unit (sequence, KV head): counts [3][chunks][kBins], above [chunks] (tokens of a
// chunk above the threshold as far as it is known, or always kept), state [4] (bins and remaining needs of the levels
// that are done).
__device__ __forceinline__ uint32_t* unit_words(const KeepLaunch& a, int s, int h) {
  return a.counts + ((int64_t)s * a.num_kv_heads + h) * keep_words(a);
}

// The thread's two bins of all chunks that have tokens
__device__ __forceinline__ void sum_bins(const uint32_t* counts, int chunks, int& c0, int& c1) {
  c0 = c1 = 0;
#pragma unroll 16
  for (int c = 0; c < chunks; ++c) {
    const uint2 x = *reinterpret_cast<const uint2*>(counts + (int64_t)c * kBins + 2 * threadIdx.x);
    c0 += (int)x.x;
    c1 += (int)x.y;
  }
}

// LEVEL 0..2: the counts of a level's bits, of the chunk's keys that begin with the bins found before
template <int LEVEL>
__global__ __launch_bounds__(kThreads) void keep_count_kernel(const KeepLaunch a) {
  __shared__ uint32_t hist[kBins * kCopies];
  __shared__ int wave_tot[kWaves], found[2];
  const int t = threadIdx.x, lane = lane_id();
  const int c = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
  const Unit u = unit_of(a, s);
  const int need = u.count - u.sink - (u.kv - u.end);
  if (need <= 0 || (int64_t)c * a.chunk >= u.kv) return;
  const int begin = c * a.chunk, end = (int)min((int64_t)u.kv, (int64_t)begin + a.chunk);
  const int chunks = (u.kv + a.chunk - 1) / a.chunk;
  uint32_t* const words = unit_words(a, s, h);
  uint32_t* const above = words + 3 * (int64_t)a.chunks * kBins;
  uint32_t* const state = above + a.chunks;
  uint32_t prefix = 0;
  if constexpr (LEVEL > 0) {
    // the bin of the level before, by every workgroup; this chunk's keys above it
    const uint32_t* before = words + (LEVEL - 1) * (int64_t)a.chunks * kBins;
    int c0, c1, bin, rest;
    sum_bins(before, chunks, c0, c1);
    find_bin(c0, c1, LEVEL == 1 ? need : (int)state[1], wave_tot, found, bin, rest);
    prefix = LEVEL == 1 ? (uint32_t)bin : state[0] << 11 | (uint32_t)bin;
    const uint2 own = *reinterpret_cast<const uint2*>(before + (int64_t)c * kBins + 2 * t);
    const int more = block_sum<kThreads>((2 * t > bin ? (int)own.x : 0) + (2 * t + 1 > bin ? (int)own.y : 0), wave_tot);
    if (t == 0) above[c] = (LEVEL == 1 ? 0u : above[c]) + (uint32_t)more;
    // (LEVEL 2 reads state[0..1] and writes state[2..3]: no workgroup changes what another reads)
    if (c == 0 && t == 0) {
      state[2 * (LEVEL - 1)] = prefix;
      state[2 * (LEVEL - 1) + 1] = (uint32_t)rest;
    }
  }
  for (int x = t; x < kBins * kCopies; x += kThreads) hist[x] = 0;
  __syncthreads();
  for (int p0 = begin + 4 * t; p0 < end; p0 += 4 * kThreads) {
    uint32_t key[4];
    load_keys(a, s, h, p0, u.kv, key);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = p0 + e;
      const bool in = p >= u.sink && p < u.end && (LEVEL == 0 || key[e] >> (LEVEL == 1 ? 21 : 10) == prefix);
      if (in) atomicAdd(&hist[bin_of(key[e], LEVEL) * kCopies + (lane & (kCopies - 1))], 1u);
    }
  }
  __syncthreads();
  uint2 sum = make_uint2(0, 0);
#pragma unroll
  for (int x = 0; x < kCopies; ++x) {
    sum.x += hist[2 * t * kCopies + x];
    sum.y += hist[(2 * t + 1) * kCopies + x];
  }
  *reinterpret_cast<uint2*>(words + (LEVEL * (int64_t)a.chunks + c) * kBins + 2 * t) = sum;
}

__global__ __launch_bounds__(kThreads) void keep_write_kernel(const KeepLaunch a) {
  __shared__ int wave_tot[kWaves], found[2];
  const int t = threadIdx.x;
  const int c = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
  const Unit u = unit_of(a, s);
  if (c == 0 && h == 0 && t == 0) a.kept[s] = u.count;
  if ((int64_t)c * a.chunk >= u.kv) return;
  const int begin = c * a.chunk, end = (int)min((int64_t)u.kv, (int64_t)begin + a.chunk);
  const int chunks = (u.kv + a.chunk - 1) / a.chunk;
  int32_t* const out = a.keep + ((int64_t)s * a.num_kv_heads + h) * a.budget;
  const int need = u.count - u.sink - (u.kv - u.end);
  // tokens before the chunk: always kept ones, ones above the threshold, ones of its key
  int gt = min(begin, u.sink) + max(begin - u.end, 0), tie = 0;
  Taken tk = {0xffffffffu, 0};
  if (need > 0) {
    const uint32_t* words = unit_words(a, s, h);
    const uint32_t* above = words + 3 * (int64_t)a.chunks * kBins;
    const uint32_t* state = above + a.chunks;
    const uint32_t* last = words + 2 * (int64_t)a.chunks * kBins;
    int c0, c1, bin, rest;
    sum_bins(last, chunks, c0, c1);
    find_bin(c0, c1, (int)state[3], wave_tot, found, bin, rest);
    tk.key = state[2] << 10 | (uint32_t)bin;
    tk.ties = rest;
    int more = 0, same = 0;
#pragma unroll 16
    for (int x = 0; x < c; ++x) {
      const uint2 own = *reinterpret_cast<const uint2*>(last + (int64_t)x * kBins + 2 * t);
      more += (2 * t > bin ? (int)own.x : 0) + (2 * t + 1 > bin ? (int)own.y : 0);
      same += 2 * t == bin ? (int)own.x : 2 * t + 1 == bin ? (int)own.y : 0;
      if (t == 0) more += (int)above[x];
    }
    gt += block_sum<kThreads>(more, wave_tot);
    tie += block_sum<kThreads>(same, wave_tot);
  }
  for (int p0 = begin; p0 < end; p0 += 4 * kThreads) {
    const int p4 = p0 + 4 * t;
    uint32_t key[4] = {0u, 0u, 0u, 0u};
    if (p4 < end) load_keys(a, s, h, p4, u.kv, key);
    bool g[4], e[4];
    int ng = 0, ne = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      classify(u, tk, p4 + i, key[i], g[i], e[i]);
      g[i] = g[i] && p4 + i < end;
      e[i] = e[i] && p4 + i < end;
      ng += g[i];
      ne += e[i];
    }
    int all_g, all_e;
    int at_g = gt + block_exclusive_scan<kThreads>(ng, wave_tot, all_g);
    int at_e = tie + block_exclusive_scan<kThreads>(ne, wave_tot, all_e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = at_g + min(at_e, tk.ties);
      if ((g[i] || (e[i] && at_e < tk.ties)) && (uint32_t)at < (uint32_t)u.count) out[at] = p4 + i;
      at_g += g[i];
      at_e += e[i];
    }
    gt += all_g;
    tie += all_e;
  }
}

// =====================================================================================
// rows to their new places
// =====================================================================================
// Row i of a sequence and KV head takes what row keep[i] holds: keys, values, their scales and the mass.  To other pages that
// is one copy.  In place rows move towards the beginning, over rows that others still have to read: all of them go to
// a stage first, and from there to their places.  A workgroup takes 64 rows, a thread 16 bytes of a row at a time, its
// loads before its stores; memory bounds it.
constexpr int kMoveRows = 64;

template <bool E4M3>
__global__ __launch_bounds__(256) void compact_kernel(const CompactLaunch a) {
  constexpr int kRowBytes = E4M3 ? kHeadDim : 2 * kHeadDim;
  constexpr int kLanes = kRowBytes / 16;                 // threads of a row
  constexpr int kSteps = kMoveRows * kLanes / 256;       // rows of a thread
  __shared__ int64_t from[kMoveRows], to[kMoveRows];
  const int t = threadIdx.x, h = blockIdx.y, s = blockIdx.z;
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  const int count = min(max(a.kept[s], 0), min(a.budget, kv));
  const int64_t unit = (int64_t)s * a.c.num_kv_heads + h, units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  const int64_t stage_rows = units * a.budget;
  char* const stage_k = a.stage;
  char* const stage_v = stage_k + stage_rows * kRowBytes;
  float* const stage_mass = reinterpret_cast<float*>(stage_v + stage_rows * kRowBytes);
  uint8_t* const stage_ks = reinterpret_cast<uint8_t*>(stage_mass + stage_rows);
  uint8_t* const stage_vs = stage_ks + stage_rows;
  const auto row_of = [&](const int32_t* table, int stride, int pos) -> int64_t {
    const int phys = phys_page(table, stride, a.c.max_pages, s, pos >> a.c.page_shift);
    return phys < 0 ? -1 : (((int64_t)h * a.c.max_pages + phys) << a.c.page_shift) + (pos & (a.c.page_size - 1));
  };
  for (int64_t i0 = (int64_t)blockIdx.x * kMoveRows; i0 < count; i0 += (int64_t)gridDim.x * kMoveRows) {
    __syncthreads();
    if (t < kMoveRows) {
      const int64_t i = i0 + t;
      int64_t f = -1, d = -1;
      if (i < count) {
        const int pos = a.keep[unit * a.budget + i];
        f = pos >= 0 && pos < kv ? row_of(a.b.page_table, a.b.table_stride, pos) : -1;
        d = a.dst_table ? row_of(a.dst_table, a.dst_stride, (int)i) : row_of(a.b.page_table, a.b.table_stride, (int)i);
        if (f < 0 || f == d) d = -1;
        if (d < 0) f = -1;
        if (a.phase == 1 && d >= 0) d = unit * a.budget + i;
        if (a.phase == 2 && f >= 0) f = unit * a.budget + i;
      }
      from[t] = f;
      to[t] = d;
    }
    __syncthreads();
    const char* const k_src = a.phase == 2 ? stage_k : static_cast<const char*>(a.c.k);
    const char* const v_src = a.phase == 2 ? stage_v : static_cast<const char*>(a.c.v);
    char* const k_dst = a.phase == 1 ? stage_k : static_cast<char*>(a.c.k);
    char* const v_dst = a.phase == 1 ? stage_v : static_cast<char*>(a.c.v);
    u32x4_t k[kSteps], v[kSteps];
    const int c = (t % kLanes) * 16;
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {  // (row 0 in place of one that does not move)
      const int64_t f = max(from[t / kLanes + x * (256 / kLanes)], (int64_t)0);
      k[x] = *reinterpret_cast<const u32x4_t*>(k_src + f * kRowBytes + c);
      v[x] = *reinterpret_cast<const u32x4_t*>(v_src + f * kRowBytes + c);
    }
    if (t < kMoveRows && from[t] >= 0) {
      const int64_t f = from[t], d = to[t];
      if (a.mass) (a.phase == 1 ? stage_mass : a.mass)[d] = (a.phase == 2 ? stage_mass : a.mass)[f];
      if constexpr (E4M3) {
        (a.phase == 1 ? stage_ks : a.c.k_scale)[d] = (a.phase == 2 ? stage_ks : a.c.k_scale)[f];
        (a.phase == 1 ? stage_vs : a.c.v_scale)[d] = (a.phase == 2 ? stage_vs : a.c.v_scale)[f];
      }
    }
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      const int64_t d = to[t / kLanes + x * (256 / kLanes)];
      if (d >= 0) {
        *reinterpret_cast<u32x4_t*>(k_dst + d * kRowBytes + c) = k[x];
        *reinterpret_cast<u32x4_t*>(v_dst + d * kRowBytes + c) = v[x];
      }
    }
  }
}

}  // namespace

void plan_keep(KeepLaunch& a) {
  a.chunks = 1;
  a.chunk = a.b.max_kv;
  if (a.b.max_kv <= kSmall) return;
  // chunks of 8192 tokens, or as many as make kMaxChunks
  a.chunk = max(8192, (int)((((int64_t)a.b.max_kv + kMaxChunks - 1) / kMaxChunks + 4095) / 4096 * 4096));
  a.chunks = (a.b.max_kv + a.chunk - 1) / a.chunk;
}

hipError_t launch_keep(const KeepLaunch& a, hipStream_t stream) {
  if (a.chunks == 1) {
    const int steps = (a.b.max_kv + 4 * kThreads - 1) / (4 * kThreads);
    const void* f = steps <= 1 ? (const void*)keep_kernel<1> : steps <= 2 ? (const void*)keep_kernel<2>
                  : steps <= 4 ? (const void*)keep_kernel<4> : (const void*)keep_kernel<8>;
    return launch_one(f, dim3(a.num_kv_heads, a.b.n_seqs), kThreads, stream, a);
  }
  const dim3 grid(a.chunks, a.num_kv_heads, a.b.n_seqs);
  for (const void* f : {(const void*)keep_count_kernel<0>, (const void*)keep_count_kernel<1>, (const void*)keep_count_kernel<2>,
                        (const void*)keep_write_kernel}) {
    const hipError_t e = launch_one(f, grid, kThreads, stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t compact_stage_bytes(const CompactLaunch& a) {
  const size_t rows = (size_t)a.b.n_seqs * a.c.num_kv_heads * a.budget;
  const size_t bytes = rows * (2 * (a.e4m3 ? 128 : 256) + 4 + (a.e4m3 ? 2 : 0));
  return (bytes + 255) / 256 * 256;
}

hipError_t launch_compact(const CompactLaunch& a, hipStream_t stream) {
  const void* f = a.e4m3 ? (const void*)compact_kernel<true> : (const void*)compact_kernel<false>;
  const int64_t units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  const int64_t rows = min(a.budget, a.b.max_kv);
  const int64_t blocks = max(min((rows + kMoveRows - 1) / kMoveRows, ((int64_t)1 << 20) / units), (int64_t)1);
  const dim3 grid((unsigned)blocks, a.c.num_kv_heads, a.b.n_seqs);
  if (a.dst_table) return launch_one(f, grid, 256, stream, a);
  CompactLaunch b = a;
  b.phase = 1;
  const hipError_t e = launch_one(f, grid, 256, stream, b);
  if (e != hipSuccess) return e;
  b.phase = 2;
  return launch_one(f, grid, 256, stream, b);
}

}  // namespace prr

// Which tokens of a cache are kept, and their rows to their new places.
#include "prr_context.h"

namespace prr {

namespace {

// =====================================================================================
// the tokens of the largest mass
// =====================================================================================
// Of a sequence and KV head: the first `sink` and the last `recent` tokens, and of those between them the ones of the largest
// mass, the lower position first among equals.  A mass becomes a 32-bit key of the same order.  Counting the keys by their
// first 11 bits finds the bin that the last token taken is in; the keys of that bin, a few hundred of 16384 where masses
// differ, are listed and counted by the next 11 and 10 bits.  So the threshold's key is known and how many of that key
// are taken, and positions come out in order: a token's place is the number of taken tokens before it.
//
// Up to 32768 tokens one workgroup does all of it, the keys in registers.  Masses share few exponents, and lanes that
// count the same bin wait for each other: there are eight counts of a bin, in banks of their own.  More tokens are cut into
// chunks of as many workgroups, in three launches: counts of each chunk in device memory; their sum, by every workgroup
// for itself, and the keys of the bin into a list; the threshold from the list, by every workgroup for itself again.
// Bound by latency: of the 13 us of 32 sequences of up to 16384 tokens and 8 KV heads, launch and keys take 4.9, the first
// count 2.6, the list and its counts 2.7, the places 3.  131072 tokens of 2 KV heads: 21 us (40 with three counts and a
// launch for each).
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 2048, kCopies = 8, kCopyPitch = kBins + 8;
constexpr int kSmall = 32768;  // tokens of one workgroup
constexpr int kMaxChunks = 64;
constexpr int kListed = 8192;  // keys of a bin that are listed in LDS

// Larger mass, larger key; NaN below everything; tokens that are kept whatever their mass above everything
constexpr uint32_t kAbsent = 0, kNaN = 1, kAlways = 0xffffffffu;
__device__ __forceinline__ uint32_t mass_key(float f) { return f != f ? kNaN : score_key(f); }
// A key that stands for a mass
__device__ __forceinline__ bool by_mass(uint32_t key) { return key - 1 < kAlways - 1; }

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
// Tokens that are chosen by their mass: at most as many as there are
__device__ __forceinline__ int chosen(const Unit& u) { return u.count - u.sink - (u.kv - u.end); }

// Where the masses of tokens [p, p + 4) lie, p a multiple of 4 below max_kv (-1: nowhere).  Needs no length, so that the
// lookup does not wait for it; what is behind the length is not used.
__device__ __forceinline__ int64_t find_keys(const KeepLaunch& a, int s, int h, int p) {
  const int phys = phys_page(a.b.page_table, a.b.table_stride, a.max_pages, s, p >> a.page_shift);
  return phys < 0 ? -1 : (((int64_t)h * a.max_pages + phys) << a.page_shift) + (p & (a.page_size - 1));
}
// Their keys; NaN where they have no page
__device__ __forceinline__ void load_keys(const KeepLaunch& a, const Unit& u, int64_t at, int p, uint32_t (&key)[4]) {
  const float nan = __builtin_nanf("");
  float4 v = make_float4(nan, nan, nan, nan);
  if (at >= 0 && p < u.kv) v = *reinterpret_cast<const float4*>(a.mass + at);
  const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    key[e] = p + e >= u.kv ? kAbsent : p + e < u.sink || p + e >= u.end ? kAlways : mass_key(f[e]);
}

struct KeepLds {
  uint32_t hist[kCopies * kCopyPitch];  // a list lies behind the first copy
  int wave_tot[kWaves], found[4], listed;
  __device__ __forceinline__ uint32_t* list() { return hist + kCopyPitch; }
};
static_assert(kListed <= (kCopies - 1) * kCopyPitch, "the list's room");
// The threshold: key, and how many tokens of it are taken
struct Taken {
  uint32_t key;
  int ties;
};

// COPIES 8: for counts of all keys; 1: of a list of few, whose lanes wait for each other for as many cycles as it has keys at most
template <int COPIES>
__device__ __forceinline__ void clear_bins(KeepLds& S) {
  for (int x = threadIdx.x; x < COPIES * kCopyPitch / 4; x += kThreads) reinterpret_cast<uint4*>(S.hist)[x] = make_uint4(0, 0, 0, 0);
  __syncthreads();
}
template <int COPIES>
__device__ __forceinline__ void count_bin(KeepLds& S, uint32_t bin) {
  atomicAdd(&S.hist[(threadIdx.x & (COPIES - 1)) * kCopyPitch + bin], 1u);
}
// Counts of the thread's two bins, 2 t and 2 t + 1, once all threads have counted
template <int COPIES>
__device__ __forceinline__ uint2 own_bins(const KeepLds& S) {
  __syncthreads();
  uint2 c = make_uint2(0, 0);
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const uint2 y = *reinterpret_cast<const uint2*>(&S.hist[x * kCopyPitch + 2 * threadIdx.x]);
    c.x += y.x;
    c.y += y.y;
  }
  return c;
}

// The bin that holds the need-th largest key, how many of the bin's keys are taken, and how many it has; c: the counts of the
// thread's two bins.  need >= 1 and at most all of them.  Calls of it have a barrier between them.
__device__ __forceinline__ void find_bin(KeepLds& S, uint2 c, int need, int& bin, int& rest, int& size) {
  const int c0 = (int)c.x, c1 = (int)c.y, t = threadIdx.x, w = t / kWave;
  const int inc = wave_inclusive_scan(c0 + c1);
  if (lane_id() == kWave - 1) S.wave_tot[w] = inc;
  __syncthreads();
  int above1 = -inc;  // keys in higher bins than the thread's
#pragma unroll
  for (int x = 0; x < kWaves; ++x) above1 += x >= w ? S.wave_tot[x] : 0;
  const int above0 = above1 + c1;
  if (above1 < need && need <= above0) {
    S.found[0] = 2 * t + 1;
    S.found[1] = need - above1;
    S.found[2] = c1;
  }
  if (above0 < need && need <= above0 + c0) {
    S.found[0] = 2 * t;
    S.found[1] = need - above0;
    S.found[2] = c0;
  }
  __syncthreads();
  bin = S.found[0];
  rest = S.found[1];
  size = S.found[2];
}

// The threshold among keys that begin with `prefix` (11 bits): the need-th largest.  each(f) calls f for the thread's part of
// them, or of keys that they are among.
template <int COPIES, class Each>
__device__ __forceinline__ Taken threshold(KeepLds& S, uint32_t prefix, int need, Each&& each) {
  int bin, size;
  clear_bins<COPIES>(S);
  each([&](uint32_t k) { if (k >> 21 == prefix) count_bin<COPIES>(S, (k >> 10) & 2047u); });
  find_bin(S, own_bins<COPIES>(S), need, bin, need, size);
  const uint32_t both = prefix << 11 | (uint32_t)bin;
  clear_bins<COPIES>(S);
  each([&](uint32_t k) { if (k >> 10 == both) count_bin<COPIES>(S, k & 1023u); });
  find_bin(S, own_bins<COPIES>(S), need, bin, need, size);
  return {both << 10 | (uint32_t)bin, need};
}

// (key > the threshold: kept for certain, 1; of the threshold's key: 2^16)
__device__ __forceinline__ uint32_t classify(const Taken& tk, uint32_t key) {
  return (key > tk.key ? 1u : 0u) + (key == tk.key ? 1u << 16 : 0u);
}
constexpr Taken kNoneByMass = {kAlways - 1, 0};

template <int ITS>
__global__ __launch_bounds__(kThreads) void keep_kernel(const KeepLaunch a) {
  __shared__ __align__(16) KeepLds S;
  __shared__ uint32_t totals[ITS * kWaves];
  const int t = threadIdx.x, lane = lane_id(), w = t / kWave;
  const int h = blockIdx.x, s = blockIdx.y;
  int64_t at[ITS];
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    const int p = it * 4 * kThreads + 4 * t;
    at[it] = p < a.b.max_kv ? find_keys(a, s, h, p) : -1;
  }
  const Unit u = unit_of(a, s);
  if (t == 0 && h == 0) a.kept[s] = u.count;
  int32_t* const out = a.keep + ((int64_t)s * a.num_kv_heads + h) * a.budget;
  if (u.count == u.kv) {
    for (int p = t; p < u.count; p += kThreads) out[p] = p;
    return;
  }
  uint32_t key[ITS][4];
#pragma unroll
  for (int it = 0; it < ITS; ++it) load_keys(a, u, at[it], it * 4 * kThreads + 4 * t, key[it]);
  Taken tk = kNoneByMass;
  int need = chosen(u);
  if (need > 0) {
    const auto each = [&](auto&& f) {
#pragma unroll
      for (int it = 0; it < ITS; ++it)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (by_mass(key[it][e])) f(key[it][e]);
    };
    int bin, size;
    if (t == 0) S.listed = 0;
    clear_bins<kCopies>(S);
    each([&](uint32_t k) { count_bin<kCopies>(S, k >> 21); });
    find_bin(S, own_bins<kCopies>(S), need, bin, need, size);
    const uint32_t prefix = (uint32_t)bin;
    if (size > kListed) {
      tk = threshold<kCopies>(S, prefix, need, each);
    } else {
      each([&](uint32_t k) {
        if (k >> 21 != prefix) return;
        const int at = atomicAdd(&S.listed, 1);
        if (at < kListed) S.list()[at] = k;
      });
      tk = threshold<1>(S, prefix, need, [&](auto&& f) {
        for (int x = t; x < size; x += kThreads) f(S.list()[x]);
      });
    }
  }
  // places: counts of each (step, wave), tokens that are taken for certain in the lower half of a word and ties in the
  // upper, then within the wave
  uint32_t inside[ITS];
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) n += classify(tk, key[it][e]);
    inside[it] = (uint32_t)wave_inclusive_scan((int)n);
    if (lane == kWave - 1) totals[it * kWaves + w] = inside[it];
    inside[it] -= n;
  }
  __syncthreads();
  // every wave adds the totals up for itself, 64 at a time
  constexpr int kSums = (ITS * kWaves + kWave - 1) / kWave;
  uint32_t before[kSums], base = 0;
#pragma unroll
  for (int x = 0; x < kSums; ++x) {
    const uint32_t n = x * kWave + lane < ITS * kWaves ? totals[x * kWave + lane] : 0u;
    const uint32_t sum = (uint32_t)wave_inclusive_scan((int)n);
    before[x] = base + sum - n;
    base += (uint32_t)__builtin_amdgcn_readlane((int)sum, kWave - 1);
  }
  const int ws = __builtin_amdgcn_readfirstlane(w);
#pragma unroll
  for (int it = 0; it < ITS; ++it) {
    uint32_t n = (uint32_t)__builtin_amdgcn_readlane((int)before[it * kWaves / kWave], it * kWaves % kWave + ws) + inside[it];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t kind = classify(tk, key[it][e]);
      const int ties = (int)(n >> 16), at = (int)(n & 0xffffu) + min(ties, tk.ties);
      if ((kind == 1 || (kind > 1 && ties < tk.ties)) && (uint32_t)at < (uint32_t)u.count) out[at] = it * 4 * kThreads + 4 * t + e;
      n += kind;
    }
  }
}

// -------------------------------------------------------------------------------------
// Several chunks.  Device memory of a unit (sequence, KV head): counts [chunks][kBins] of the first bits; above [chunks], a
// chunk's keys in higher bins than the threshold's; state [4]: the length of the list, the threshold's bin, the keys of
// it that are taken; list [chunks * chunk] (key, chunk), in any order.
struct UnitWords {
  uint32_t* counts;
  uint32_t* above;
  uint32_t* state;
  uint2* list;
};
__device__ __forceinline__ UnitWords unit_words(const KeepLaunch& a, int s, int h) {
  UnitWords w;
  w.counts = a.counts + ((int64_t)s * a.num_kv_heads + h) * keep_words(a);
  w.above = w.counts + (int64_t)a.chunks * kBins;
  w.state = w.above + kMaxChunks;
  w.list = reinterpret_cast<uint2*>(w.state + 4);
  return w;
}

struct Chunk {
  int c, h, s, begin, end, chunks;
};
__device__ __forceinline__ Chunk chunk_of(const KeepLaunch& a, const Unit& u) {
  Chunk r;
  r.c = blockIdx.x;
  r.h = blockIdx.y;
  r.s = blockIdx.z;
  r.begin = (int)min((int64_t)r.c * a.chunk, (int64_t)u.kv);
  r.end = (int)min((int64_t)r.begin + a.chunk, (int64_t)u.kv);
  r.chunks = (u.kv + a.chunk - 1) / a.chunk;
  return r;
}

__global__ __launch_bounds__(kThreads) void keep_count_kernel(const KeepLaunch a) {
  __shared__ __align__(16) KeepLds S;
  const int t = threadIdx.x;
  const Unit u = unit_of(a, blockIdx.z);
  const Chunk k = chunk_of(a, u);
  if (chosen(u) <= 0 || k.begin >= k.end) return;
  const UnitWords m = unit_words(a, k.s, k.h);
  if (k.c == 0 && t == 0) m.state[0] = 0;
  clear_bins<kCopies>(S);
#pragma unroll 2
  for (int p0 = k.begin + 4 * t; p0 < k.end; p0 += 4 * kThreads) {
    uint32_t key[4];
    load_keys(a, u, find_keys(a, k.s, k.h, p0), p0, key);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (by_mass(key[e])) count_bin<kCopies>(S, key[e] >> 21);
  }
  *reinterpret_cast<uint2*>(m.counts + (int64_t)k.c * kBins + 2 * t) = own_bins<kCopies>(S);
}

__global__ __launch_bounds__(kThreads) void keep_list_kernel(const KeepLaunch a) {
  __shared__ __align__(16) KeepLds S;
  const int t = threadIdx.x, lane = lane_id();
  const Unit u = unit_of(a, blockIdx.z);
  const Chunk k = chunk_of(a, u);
  const int need = chosen(u);
  if (need <= 0 || k.begin >= k.end) return;
  const UnitWords m = unit_words(a, k.s, k.h);
  // the chunk's first keys are on their way while the counts are added up
  const int p1 = k.begin + 4 * t;
  uint32_t key[4] = {kAbsent, kAbsent, kAbsent, kAbsent};
  if (p1 < k.end) load_keys(a, u, find_keys(a, k.s, k.h, p1), p1, key);
  const uint2 own = *reinterpret_cast<const uint2*>(m.counts + (int64_t)k.c * kBins + 2 * t);
  uint2 sum = make_uint2(0, 0);
#pragma unroll 16
  for (int c = 0; c < k.chunks; ++c) {
    const uint2 x = *reinterpret_cast<const uint2*>(m.counts + (int64_t)c * kBins + 2 * t);
    sum.x += x.x;
    sum.y += x.y;
  }
  int bin, rest, size;
  find_bin(S, sum, need, bin, rest, size);
  __syncthreads();
  const int above = block_sum<kThreads>((2 * t > bin ? (int)own.x : 0) + (2 * t + 1 > bin ? (int)own.y : 0), S.wave_tot);
  if (t == 0) {
    m.above[k.c] = (uint32_t)above;
    if (k.c == 0) {
      m.state[1] = (uint32_t)bin;
      m.state[2] = (uint32_t)rest;
    }
  }
  if (2 * t == (bin & ~1)) S.listed = (int)atomicAdd(&m.state[0], bin & 1 ? own.y : own.x);  // this chunk's part of the list
  __syncthreads();
  for (int p0 = p1; p0 - 4 * t < k.end; p0 += 4 * kThreads) {
    if (p0 != p1 && p0 < k.end) load_keys(a, u, find_keys(a, k.s, k.h, p0), p0, key);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = p0 < k.end && by_mass(key[e]) && key[e] >> 21 == (uint32_t)bin;
      const uint64_t all = __ballot(in);
      if (!all) continue;
      int base = 0;
      if (lane == 0) base = atomicAdd(&S.listed, (int)__popcll(all));
      base = __builtin_amdgcn_readfirstlane(base) + lanes_below(all);
      if (in && (uint32_t)base < (uint32_t)(a.chunks * (int64_t)a.chunk)) m.list[base] = make_uint2(key[e], (uint32_t)k.c);
    }
  }
}

__global__ __launch_bounds__(kThreads) void keep_write_kernel(const KeepLaunch a) {
  __shared__ __align__(16) KeepLds S;
  const int t = threadIdx.x;
  const Unit u = unit_of(a, blockIdx.z);
  const Chunk k = chunk_of(a, u);
  if (k.c == 0 && k.h == 0 && t == 0) a.kept[k.s] = u.count;
  if (k.begin >= k.end) return;
  int32_t* const out = a.keep + ((int64_t)k.s * a.num_kv_heads + k.h) * a.budget;
  // tokens before the chunk: always kept ones, ones above the threshold, ones of its key
  int gt = min(k.begin, u.sink) + max(k.begin - u.end, 0), tie = 0;
  Taken tk = kNoneByMass;
  const int p1 = k.begin + 4 * t;
  uint32_t key[4] = {kAbsent, kAbsent, kAbsent, kAbsent};
  if (p1 < k.end) load_keys(a, u, find_keys(a, k.s, k.h, p1), p1, key);
  if (chosen(u) > 0) {
    const UnitWords m = unit_words(a, k.s, k.h);
    const int n = (int)min((int64_t)m.state[0], a.chunks * (int64_t)a.chunk);
    const int need = (int)m.state[2];
    const int above = t < k.c ? (int)m.above[t] : 0;  // (at most 64 chunks)
    const uint32_t prefix = m.state[1];
    int g = above, e = 0;
    if (n <= kListed) {
      for (int x = t; x < n; x += kThreads) S.list()[x] = m.list[x].x;
      tk = threshold<1>(S, prefix, need, [&](auto&& f) {
        for (int x = t; x < n; x += kThreads) f(S.list()[x]);
      });
    } else {
      tk = threshold<kCopies>(S, prefix, need, [&](auto&& f) {
#pragma unroll 4
        for (int x = t; x < n; x += kThreads) f(m.list[x].x);
      });
    }
#pragma unroll 4
    for (int x = t; x < n; x += kThreads) {
      const uint2 y = m.list[x];
      const bool before = (int)y.y < k.c;
      g += before && y.x > tk.key;
      e += before && y.x == tk.key;
    }
    __syncthreads();
    gt += block_sum<kThreads>(g, S.wave_tot);
    tie += block_sum<kThreads>(e, S.wave_tot);
  }
  for (int p0 = k.begin; p0 < k.end; p0 += 4 * kThreads) {
    const int p4 = p0 + 4 * t;
    if (p0 != k.begin && p4 < k.end) load_keys(a, u, find_keys(a, k.s, k.h, p4), p4, key);
    uint32_t kind[4], n = 0;  // (at most 4096 of each in a step)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kind[i] = p4 < k.end ? classify(tk, key[i]) : 0;
      n += kind[i];
    }
    int all;
    const int before = block_exclusive_scan<kThreads>((int)n, S.wave_tot, all);
    int at_g = gt + (before & 0xffff), at_e = tie + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = at_g + min(at_e, tk.ties);
      if ((kind[i] == 1 || (kind[i] > 1 && at_e < tk.ties)) && (uint32_t)at < (uint32_t)u.count) out[at] = p4 + i;
      at_g += (int)(kind[i] & 1);
      at_e += (int)(kind[i] >> 16);
    }
    gt += all & 0xffff;
    tie += all >> 16;
  }
}

// =====================================================================================
// rows to their new places
// =====================================================================================
// Row i of a sequence and KV head takes what row keep[i] holds: keys, values, their scales and the mass.  To other pages that
// is one copy.  In place rows move towards the beginning, over rows that others still have to read: all of them go to
// a stage first, and from there to their places.  A workgroup takes 64 rows, a thread 16 bytes of a row at a time, its
// loads before its stores; memory bounds it.  What is not a stage passes the caches by: 32 sequences of 2048 e4m3 tokens,
// 8 KV heads, from cold memory 59 us, 4.6 TB/s (68 by way of the caches); in place 94 to 101.
constexpr int kMoveRows = 64;

// PHASE 0: to other pages, 1: to the stage, 2: from the stage
template <bool E4M3, int PHASE>
__global__ __launch_bounds__(256) void compact_kernel(const CompactLaunch a) {
  constexpr int kRowBytes = E4M3 ? kHeadDim : 2 * kHeadDim;
  constexpr int kLanes = kRowBytes / 16;                 // threads of a row
  constexpr int kSteps = kMoveRows * kLanes / 256;       // rows of a thread
  __shared__ int64_t from[kMoveRows], to[kMoveRows];
  const int t = threadIdx.x, h = blockIdx.y, s = blockIdx.z;
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  const int count = min(max(a.kept[s], 0), min(a.budget, kv));
  const int64_t unit = (int64_t)s * a.c.num_kv_heads + h, units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  const int64_t stage_row = unit * a.stage_rows, stage_rows = units * a.stage_rows;
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
        if (PHASE == 1 && d >= 0) d = stage_row + i;
        if (PHASE == 2 && f >= 0) f = stage_row + i;
      }
      from[t] = f;
      to[t] = d;
    }
    __syncthreads();
    const char* const k_src = PHASE == 2 ? stage_k : static_cast<const char*>(a.c.k);
    const char* const v_src = PHASE == 2 ? stage_v : static_cast<const char*>(a.c.v);
    char* const k_dst = PHASE == 1 ? stage_k : static_cast<char*>(a.c.k);
    char* const v_dst = PHASE == 1 ? stage_v : static_cast<char*>(a.c.v);
    u32x4_t k[kSteps], v[kSteps];
    const int c = (t % kLanes) * 16;
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {  // (row 0 in place of one that does not move)
      const int64_t f = max(from[t / kLanes + x * (256 / kLanes)], (int64_t)0);
      const auto* const kp = reinterpret_cast<const u32x4_t*>(k_src + f * kRowBytes + c);
      const auto* const vp = reinterpret_cast<const u32x4_t*>(v_src + f * kRowBytes + c);
      k[x] = PHASE == 2 ? *kp : __builtin_nontemporal_load(kp);
      v[x] = PHASE == 2 ? *vp : __builtin_nontemporal_load(vp);
    }
    if (t < kMoveRows && from[t] >= 0) {
      const int64_t f = from[t], d = to[t];
      if (a.mass) (PHASE == 1 ? stage_mass : a.mass)[d] = (PHASE == 2 ? stage_mass : a.mass)[f];
      if constexpr (E4M3) {
        (PHASE == 1 ? stage_ks : a.c.k_scale)[d] = (PHASE == 2 ? stage_ks : a.c.k_scale)[f];
        (PHASE == 1 ? stage_vs : a.c.v_scale)[d] = (PHASE == 2 ? stage_vs : a.c.v_scale)[f];
      }
    }
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      const int64_t d = to[t / kLanes + x * (256 / kLanes)];
      if (d >= 0) {
        auto* const kp = reinterpret_cast<u32x4_t*>(k_dst + d * kRowBytes + c);
        auto* const vp = reinterpret_cast<u32x4_t*>(v_dst + d * kRowBytes + c);
        if constexpr (PHASE == 1) {
          *kp = k[x];
          *vp = v[x];
        } else {
          __builtin_nontemporal_store(k[x], kp);
          __builtin_nontemporal_store(v[x], vp);
        }
      }
    }
  }
}

// The mass of places without a token: positions from `from` to the end of the sequence's last page, one thread a position.
// Memory and the launch bound it: 32 sequences of up to 16384 tokens, 8 KV heads, to 2048: 7.5 us;
// one of 5000 to 1000 4.0.
__global__ __launch_bounds__(256) void mass_clear_kernel(const MassClearLaunch a) {
  const int h = blockIdx.y, s = blockIdx.z;
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  const int from = min(max(a.from[s], 0), kv);
  const int64_t end = ((int64_t)kv + a.page_size - 1) >> a.page_shift << a.page_shift;
  for (int64_t p = from + (int64_t)blockIdx.x * 256 + threadIdx.x; p < end; p += (int64_t)gridDim.x * 256) {
    const int phys = phys_page(a.b.page_table, a.b.table_stride, a.max_pages, s, (int)(p >> a.page_shift));
    if (phys >= 0) a.mass[(((int64_t)h * a.max_pages + phys) << a.page_shift) + (p & (a.page_size - 1))] = 0.0f;
  }
}

}  // namespace

hipError_t launch_mass_clear(const MassClearLaunch& a, hipStream_t stream) {
  const int64_t units = (int64_t)a.b.n_seqs * a.num_kv_heads;
  const int64_t blocks = max(min(((int64_t)a.b.max_kv + a.page_size + 255) / 256, ((int64_t)1 << 18) / units), (int64_t)1);
  return launch_one((const void*)mass_clear_kernel, dim3((unsigned)blocks, a.num_kv_heads, a.b.n_seqs), 256, stream, a);
}

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
  for (const void* f : {(const void*)keep_count_kernel, (const void*)keep_list_kernel, (const void*)keep_write_kernel}) {
    const hipError_t e = launch_one(f, grid, kThreads, stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t compact_stage_bytes(const CompactLaunch& a) {
  const size_t rows = (size_t)a.b.n_seqs * a.c.num_kv_heads * a.stage_rows;
  const size_t bytes = rows * (2 * (a.e4m3 ? 128 : 256) + 4 + (a.e4m3 ? 2 : 0));
  return (bytes + 255) / 256 * 256;
}

hipError_t launch_compact(const CompactLaunch& a, hipStream_t stream) {
  const int64_t units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  const int64_t rows = a.stage_rows;
  const int64_t blocks = max(min((rows + kMoveRows - 1) / kMoveRows, ((int64_t)1 << 20) / units), (int64_t)1);
  const dim3 grid((unsigned)blocks, a.c.num_kv_heads, a.b.n_seqs);
  if (a.dst_table)
    return launch_one(a.e4m3 ? (const void*)compact_kernel<true, 0> : (const void*)compact_kernel<false, 0>, grid, 256, stream, a);
  const hipError_t e = launch_one(a.e4m3 ? (const void*)compact_kernel<true, 1> : (const void*)compact_kernel<false, 1>, grid, 256,
                                  stream, a);
  if (e != hipSuccess) return e;
  return launch_one(a.e4m3 ? (const void*)compact_kernel<true, 2> : (const void*)compact_kernel<false, 2>, grid, 256, stream, a);
}

}  // namespace prr
